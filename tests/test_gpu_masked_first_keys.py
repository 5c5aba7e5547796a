"""Keys that count nothing at the start of the context, where the attention kernels take their first reference: whole 32-key blocks and tiles of them,
from infinite components and from finite ones whose scores overflow, for all query heads or for every other one."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2605_06472_amd import binding, workloads as W          # noqa: E402
from tests.gpu_util import DeviceBatch, assert_close               # noqa: E402

HEADS = [(32, 8, 128), (16, 2, 64), (4, 4, 64)]


def _bits(x):
    return W.f32_to_bf16_bits(np.full(1, x, np.float32))[0]


def _batch(seed, heads, first, kind):
    """`first` tokens that count nothing, in the prefix or, where that is shorter, in the suffix as well.  kind: "infinite" (and every other score
    near -650 in log2 units), "overflow", "some" (the same, for even query heads only)."""
    hq, hkv, d = heads
    prefix = 300 if first <= 200 else 1100
    b = W.ragged_small(seed, "bf16", Hq=hq, Hkv=hkv, d=d, prefix_lens=(prefix, 0), new_lens=(70, 300), num_pages=150)
    b.q[:, :, 0] = _bits(32.0)
    keys = [(b.kv_pool, (slice(None), 0)), (b.k_new, (slice(None),))]
    for a, at in keys:
        a[at + (..., 0)] = 0
    if kind == "infinite":
        b.q[:, :, 1] = _bits(16.0)
        for a, at in keys:
            a[at + (..., 1)] = _bits(-320.0 if d == 64 else -448.0)
    if kind == "some":
        b.q[:, 1::2, 0] = 0
    nothing = _bits(-np.inf if kind == "infinite" else -3e38)
    for t in range(first):
        b.kv_pool[b.block_table[0, t // 16], 0, :, t % 16, 0] = nothing
    b.k_new[70:70 + first, :, 0] = nothing
    return b


@pytest.mark.parametrize("kind", ["infinite", "overflow", "some"])
@pytest.mark.parametrize("first", [16, 32, 40, 64, 96, 200])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
def test_the_first_keys_count_nothing(oracle, heads, first, kind):
    b = _batch(910 + first, heads, first, kind)
    want = oracle.prefill(b.q, b.k_new, b.v_new, b.kv_pool, b.block_table, b.prefix_lens, b.new_lens)
    rows = np.r_[0:70, 70 + first:370]                             # (rows before see nothing, and have no value)
    assert np.isfinite(want[rows]).all()
    db = DeviceBatch(b)
    got = {}
    for waves in (0, 4, 8, 64):
        binding.set_attn_waves(waves)
        try:
            db.out.fill_(7.0)
            db.prefill()
            torch.cuda.synchronize()
        finally:
            binding.set_attn_waves(0)
        got[waves] = db.out_f64()[rows]
        assert_close(got[waves], want[rows], "bf16", "%s %s, %d waves" % (kind, heads, waves))
    assert np.array_equal(got[4], got[8]) and np.array_equal(got[4], got[64])
