"""A NaN among the scores of a decode row over a bf16 pool, or an infinite one, makes the row NaN, as it does in the prefill; a row
without tokens, or with scores of minus infinity alone, is zero."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2605_06472_amd import binding, workloads as W          # noqa: E402
from tests.gpu_util import DeviceBatch                             # noqa: E402

HEADS = [(8, 2, 128), (16, 2, 64), (16, 2, 128), (32, 2, 128), (4, 4, 64)]
NAN, INF = 0x7fc0, 0x7f80
CONTEXTS = (4097, 40, 1003)                     # in several slices (the last a token), whole


def decoded(b):
    db = DeviceBatch(b)
    got = []
    for entry in (binding.paged_decode, binding.paged_decode_static):
        out = torch.full_like(db.q, 7.0)
        entry(db.shape, db.q, db.kv_pool, db.block_table, b.prefix_lens, out)
        got.append(out)
    torch.cuda.synchronize()
    assert torch.equal(got[0].view(torch.int16), got[1].view(torch.int16))
    return got[0].float()


def bf16(x):
    return W.f32_to_bf16_bits(np.full(1, x, np.float32))[0]


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
def test_a_bad_key_shows(heads):
    hq, hkv, d = heads
    per = hq // hkv
    b = W.ragged_small(330, "bf16", Hq=hq, Hkv=hkv, d=d, prefix_lens=CONTEXTS, new_lens=(1,) * 3, num_pages=400)
    want = decoded(b)
    for bits in (NAN, INF):
        for request, token in ((0, 4096), (0, 77), (1, 0), (1, 39), (2, 500)):
            if bits == INF:
                b.q[request, per, 5] = bf16(1.0)             # (one query head at least whose score is plus infinity)
                want = decoded(b)
            page, slot = b.block_table[request, token // 16], token % 16
            was = b.kv_pool[page, 0, 1, slot, 5]
            b.kv_pool[page, 0, 1, slot, 5] = bits
            got = decoded(b)
            b.kv_pool[page, 0, 1, slot, 5] = was
            rows = slice(per, 2 * per) if bits == NAN else slice(per, per + 1)
            assert bool(torch.isnan(got[request, rows]).all()), (bits, request, token)
            got[request, per:2 * per] = want[request, per:2 * per]
            assert torch.equal(got, want)


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
def test_an_infinite_or_nan_query_shows(heads):
    hq, hkv, d = heads
    per = hq // hkv
    b = W.ragged_small(331, "bf16", Hq=hq, Hkv=hkv, d=d, prefix_lens=CONTEXTS, new_lens=(1,) * 3, num_pages=400)
    want = decoded(b)
    for bits in (INF, INF | 0x8000, NAN):
        b.q[:, 1, 9] = bits
        got = decoded(b)
        assert bool(torch.isnan(got[:, 1]).all()) and bool(torch.isfinite(got[:, 0]).all())
        assert torch.equal(got[:, max(per, 2):], want[:, max(per, 2):])


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
def test_nothing_counts(heads):
    """No tokens, or scores that all overflow to minus infinity: zeros."""
    hq, hkv, d = heads
    b = W.ragged_small(332, "bf16", Hq=hq, Hkv=hkv, d=d, prefix_lens=(4097, 0, 1003, 17), new_lens=(1,) * 4, num_pages=400)
    b.q[:] = bf16(2.0)
    used = b.block_table[0, :257]
    b.kv_pool[used, 0] = bf16(-3e38)
    b.kv_pool[b.block_table[3, :2], 0] = bf16(-3e38)
    got = decoded(b)
    assert not bool(got[[0, 1, 3]].any()) and bool(torch.isfinite(got[2]).all()) and bool(got[2].any())
