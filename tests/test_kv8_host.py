"""The 8-bit pool at the C boundary without a GPU: what is refused, and what the host decides and launches."""
import numpy as np
import pytest

from paper_2605_06472_amd import binding
from tests.test_abi_host import FAKE, _shape
from tests.test_host_routes import _covers, fake_runtime, over_fake      # noqa: F401

I32 = np.int32


def _code(call, *args, **kw):
    with pytest.raises(binding.PbkvError) as e:
        call(*args, **kw)
    assert str(e.value)
    return e.value.code


def _read(shape, first, num, pool=FAKE, k=FAKE, v=FAKE, table=FAKE):
    binding.read_kv(shape, pool, table, np.array(first, I32), np.array(num, I32), k, v, stream=0)


def test_page_bytes():
    assert binding.page_bytes(_shape(dtype="bf16_kv8")) == 33024
    assert binding.page_bytes(_shape(num_q_heads=1, num_kv_heads=1, head_dim=64, dtype="bf16_kv8")) == 2176      # 2080 in whole lines
    assert binding.page_bytes(_shape(head_dim=96, dtype="bf16_kv8")) == 0
    assert binding.make_shape(1, 1, 1, 64, 16, 1, 1, "bf16_kv8").dtype == 2


@pytest.mark.parametrize("dtype", ["bf16", "f32", "bf16_kv8"])
def test_read_refuses_what_append_does(dtype):
    s = _shape(batch=2, dtype=dtype)
    assert _code(_read, s, [0, 0], [16, 16], pool=None) == -1
    assert _code(_read, s, [0, 0], [16, 16], k=None) == -1
    assert _code(_read, s, [0, 0], [16, 16], v=None) == -1
    assert _code(_read, s, [0, 0], [16, 16], table=None) == -1
    assert _code(_read, s, [0, -1], [16, 16]) == -4
    assert _code(_read, s, [0, 0], [16, -1]) == -4
    assert _code(_read, s, [0, 100], [16, 29]) == -4
    assert _code(_read, s, [0, 0], [16, 16], k=FAKE + 8) == -2
    assert _code(_read, s, [0, 0], [16, 16], pool=FAKE + 8) == -2
    assert _code(_read, s, [0, 0], [16, 16]) == -6                              # no device memory
    assert _code(_read, _shape(dtype=dtype, page_size=32), [0], [1]) == -2
    assert _code(_read, _shape(dtype=3), [0], [1]) == -3
    _read(_shape(batch=0, dtype=dtype), [], [])
    _read(s, [5, 0], [0, 0])


def test_what_else_is_refused():
    s = _shape(dtype="bf16_kv8")
    assert _code(binding.append_kv, s, FAKE, FAKE, FAKE, FAKE, np.array([-1], I32), np.array([1], I32), stream=0) == -4
    assert _code(binding.prefix_prefill, s, FAKE, FAKE, FAKE, FAKE, FAKE, np.array([16], I32), np.array([16], I32), FAKE, stream=0) == -6
    assert _code(binding.prefix_prefill, _shape(num_q_heads=24, dtype="bf16_kv8"), FAKE, FAKE, FAKE, FAKE, FAKE, np.array([16], I32), np.array([16], I32), FAKE, stream=0) == -2
    for call in (binding.paged_decode, binding.paged_decode_static):
        assert _code(call, s, FAKE, FAKE, FAKE, np.array([1000], I32), FAKE, stream=0) == -4
        assert _code(call, s, FAKE, None, FAKE, np.array([10], I32), FAKE, stream=0) == -1
        assert _code(call, _shape(num_q_heads=24, dtype="bf16_kv8"), FAKE, FAKE, FAKE, np.array([10], I32), FAKE, stream=0) == -2
    assert _code(binding.gather_probe, s, FAKE, FAKE, FAKE, FAKE, np.array([16], I32), np.array([16], I32), None, stream=0) == -3
    assert _code(binding.swap_in_pages, s, FAKE, np.array([1, 64], I32), FAKE, stream=0) == -4
    # the largest pool: 512 GiB
    pages = (1 << 39) // 33024
    assert _code(_read, _shape(num_pages=pages, dtype="bf16_kv8"), [0], [16]) == -6
    assert _code(_read, _shape(num_pages=pages + 1, dtype="bf16_kv8"), [0], [16]) == -7
    # the largest page: 2 GiB
    heads = (1 << 31) // (32 * 129)
    assert _code(_read, _shape(num_q_heads=heads, num_kv_heads=heads, num_pages=1, dtype="bf16_kv8"), [0], [16]) == -6
    assert _code(_read, _shape(num_q_heads=heads + 1, num_kv_heads=heads + 1, num_pages=1, dtype="bf16_kv8"), [0], [16]) == -7
    assert _code(_read, _shape(num_q_heads=1 << 18, num_kv_heads=1 << 18, num_pages=1), [0], [16]) == -7


# ---- over the recording runtime ----------------------------------------------------------------------------------
def _call(prefix, new, hq=32, hkv=8, d=128, stream=0):
    shape = binding.make_shape(len(new), hq, hkv, d, 16, 4096, 1 << 20, "bf16_kv8")
    binding.prefix_prefill(shape, FAKE, FAKE, FAKE, FAKE, FAKE, np.asarray(prefix, I32), np.asarray(new, I32), FAKE, stream=stream)


def check_prefill_routes(fake):
    """Whole, cut and 64-row launches cover every tile, the second call from the list that the first one left; the bf16 call of the same
    lengths between them takes its own list and kernels."""
    for prefix, new, kw in (([300, 77, 0], [130, 65, 70], {}), ([4000, 7], [33, 5], {}), ([32768] * 4, [2048] * 4, {}), ([900, 3], [40, 700], dict(hq=16, hkv=2, d=64))):
        for call in range(2):
            fake.forget()
            _call(prefix, new, **kw)
            main, merge = fake.launches("attn_bf16"), fake.launches("merge")
            assert len(main) == 1 and "Lb1EEEv" in main[0]["name"], main[0]["name"]
            _covers(main, merge, prefix, new, **{k: v for k, v in kw.items() if k != "d"})
            fake.forget()
            shape = binding.make_shape(len(new), kw.get("hq", 32), kw.get("hkv", 8), kw.get("d", 128), 16, 4096, 1 << 20, "bf16")
            binding.prefix_prefill(shape, FAKE, FAKE, FAKE, FAKE, FAKE, np.asarray(prefix, I32), np.asarray(new, I32), FAKE, stream=0)
            (plain,) = fake.launches("attn_bf16")
            assert "Lb0EEEv" in plain["name"]


def test_prefill_routes(over_kv8):
    over_kv8("check_prefill_routes")


def check_decode_routes(fake):
    """The one-kernel form, the one with a merge kernel, and lists in memory, by their kernels' names."""
    def run(ctx, hq=32, hkv=8, d=128, static=False):
        fake.forget()
        shape = binding.make_shape(len(ctx), hq, hkv, d, 16, 4096, 1 << 20, "bf16_kv8")
        (binding.paged_decode_static if static else binding.paged_decode)(shape, FAKE, FAKE, FAKE, np.asarray(ctx, I32), FAKE, stream=0)
        return fake.launches("decode_")
    (one,) = run([5000])
    assert "decode_kv8_kernelILi128ELb1ELb1E" in one["name"] and one["counters"]
    main, merge = run([5000], static=True)
    assert "decode_kv8_kernelILi128ELb0ELb1E" in main["name"] and "merge" in merge["name"]
    (many,) = run([40] * 300, hq=16, hkv=2, d=64)
    assert "decode_kv8_kernelILi64E" in many["name"] and "ELb0EEEv" in many["name"] and many["list"]
    (again,) = run([40] * 300, hq=16, hkv=2, d=64)
    assert again["list"] != many["list"]                     # the copy that the first launch left in device memory


def test_decode_routes(over_kv8):
    over_kv8("check_decode_routes")


@pytest.fixture
def over_kv8(fake_runtime):                                   # noqa: F811
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

    def run(check):
        code = ("import sys; sys.path.insert(0, %r); from tests.host.fake import Fake; fake = Fake(%r); from tests import test_kv8_host as t; t.%s(fake); print('clean')"
                % (root, fake_runtime, check))
        r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=root)
        assert r.returncode == 0 and r.stdout.strip().endswith("clean"), (r.stdout + r.stderr)[-3000:]
    return run
