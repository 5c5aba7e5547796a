"""A NaN key makes every row that attends to it NaN in the prefill, over bf16 and 8-bit pools: in a launch of one range, of many ranges whose partial results
are merged, with two key groups, and where the NaN's range weighs nothing."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2605_06472_amd import binding, workloads as W          # noqa: E402
from tests.kv8_util import DeviceKv8, make                         # noqa: E402

NAN = 0x7fc0


@pytest.mark.parametrize("plain", [True, False], ids=["bf16", "kv8"])
@pytest.mark.parametrize("heads", [(8, 2, 128), (16, 2, 64), (4, 4, 64)], ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("prefix,new", [((4097, 40), (33, 20)), ((700, 2000), (300, 129))], ids=["cut", "whole"])
def test_a_nan_key_shows(prefix, new, heads, plain):
    hq, hkv, d = heads
    per = hq // hkv
    b = W.ragged_small(350, "bf16", Hq=hq, Hkv=hkv, d=d, prefix_lens=prefix, new_lens=new, num_pages=400)
    # the first 64 pages of the first request score 900 below the rest in log2 units
    b.q[:new[0], :, 1] = W.f32_to_bf16_bits(np.full(1, 16, np.float32))[0]
    b.kv_pool[b.block_table[0, :min(64, prefix[0] // 32)], 0, :, :, 1] = W.f32_to_bf16_bits(np.full(1, -448, np.float32))[0]

    def results():
        # (a pool's values from their 8-bit form for both)
        dev, got = DeviceKv8(make(b)), []
        try:
            for waves in (0, 4, 8, 64):
                binding.set_attn_waves(waves)
                got.append(dev.prefill(plain=plain).float())
        finally:
            binding.set_attn_waves(0)
        return got

    want = results()
    assert all(bool(torch.isfinite(w).all()) for w in want)
    head = slice(per, 2 * per)
    for request, token in ((0, 5), (0, prefix[0] - 1), (1, 17)):
        page, slot = b.block_table[request, token // 16], token % 16
        was = b.kv_pool[page, 0, 1, slot, 5]
        b.kv_pool[page, 0, 1, slot, 5] = NAN
        rows = slice(0, new[0]) if request == 0 else slice(new[0], sum(new))
        for got, w in zip(results(), want):
            assert bool(torch.isnan(got[rows, head]).all())
            got[rows, head] = w[rows, head]
            assert torch.equal(got, w)
        b.kv_pool[page, 0, 1, slot, 5] = was
