"""A NaN among the scores of a decode row over an 8-bit pool makes the row NaN, whichever slice of the context it stands in and however little that
slice weighs: alone in its slice, far below the scores of the others, or in every slice."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2605_06472_amd import workloads as W                                  # noqa: E402
from tests.kv8_util import DeviceKv8, make                                       # noqa: E402

# 4097 tokens are 256 pages and a token: the last slice is that token alone, in slices of any power of two of pages; in 64-page ones or shorter
# eight and sixteen heads of 128 have more partials than one work-group holds, and a kernel of several merges them
HEADS = [(8, 2, 128), (16, 2, 64), (16, 2, 128), (32, 2, 128), (4, 4, 64)]
NAN, INF = 0x7fc0, 0x7f80


def decoded(b):
    d = DeviceKv8(make(b))
    got = [d.decode(), d.decode(static=True)]
    torch.cuda.synchronize()
    assert torch.equal(got[0].view(torch.int16), got[1].view(torch.int16))
    return got[0].float()


def batch(seed, heads):
    hq, hkv, d = heads
    return W.ragged_small(seed, "bf16", Hq=hq, Hkv=hkv, d=d, prefix_lens=(4097, 40, 1003), new_lens=(1,) * 3, num_pages=400)


def check(b, want, heads, head=1):
    got, per = decoded(b), heads[0] // heads[1]
    rows = slice(head * per, (head + 1) * per)
    assert bool(torch.isnan(got[0, rows]).all())
    got[0, rows] = want[0, rows]
    assert torch.equal(got, want)                            # no other row is touched


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("bits", [NAN, INF], ids=["nan", "inf"])
def test_a_slice_of_nothing_else(heads, bits):
    b = batch(320, heads)
    want = decoded(b)
    assert bool(torch.isfinite(want).all())
    for token in (4096, 0, 2000):
        page, slot = b.block_table[0, token // 16], token % 16
        was = b.kv_pool[page, 0, 1, slot].copy()
        b.kv_pool[page, 0, 1, slot, 5] = bits
        check(b, want, heads)
        b.kv_pool[page, 0, 1, slot] = was


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
def test_slices_that_weigh_nothing(heads):
    """The first half of the context scores 900 below the other in log2 units, and holds the NaN."""
    b = batch(321, heads)
    b.q[0, :, 1] = W.f32_to_bf16_bits(np.full(1, 16, np.float32))[0]
    b.kv_pool[b.block_table[0, :129], 0, :, :, 1] = W.f32_to_bf16_bits(np.full(1, -448, np.float32))[0]
    want = decoded(b)
    assert bool(torch.isfinite(want).all())
    b.kv_pool[b.block_table[0, 3], 0, 1, 7, 5] = NAN
    check(b, want, heads)


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
def test_infinite_scores_in_every_slice(heads):
    """An infinite query component: scores of plus and minus infinity all over the context, of one query head."""
    b = batch(322, heads)
    want = decoded(b)
    for bits in (INF, INF | 0x8000, NAN):
        b.q[0, 1, 9] = bits
        got = decoded(b)
        assert bool(torch.isnan(got[0, 1]).all())
        got[0, 1] = want[0, 1]
        # Heads of the same KV head move their references at other pages then: each side is off by its probabilities' 2^-17 and as much again of fp32
        # sums, times the largest |v| (5), before a rounding to bf16 that may fall on either side of a step (2^-7 of the value).
        assert bool(((got - want).abs() <= 2.0 ** -7 * want.abs() + 2 * 2.0 ** -16 * 5).all())
        per = heads[0] // heads[1]
        assert torch.equal(got[1:], want[1:]) and torch.equal(got[0, max(per, 2):], want[0, max(per, 2):])
