"""Pages of an 8-bit pool as callers may name them: ids outside the pool, which every kernel clamps, and a last prefix page whose free slots an
append on another stream fills while a prefill reads the others."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import kv8_oracle as K8                                              # noqa: E402
from paper_2605_06472_amd import binding, workloads as W                         # noqa: E402
from tests.gpu_util import to_torch                                              # noqa: E402
from tests.kv8_util import DeviceKv8, make                                       # noqa: E402


def full_pool(b):
    """Every slot of every page holds a row."""
    pool = np.zeros((b.num_pages, K8.page_bytes(b.Hkv, b.d)), np.uint8)
    codes, scales = K8.quantise(b.kv_pool)
    K8.codes_of(pool, b.Hkv, b.d)[:], K8.scales_of(pool, b.Hkv, b.d)[:] = codes, np.moveaxis(scales, 1, -1)
    return pool


@pytest.mark.parametrize("heads", [(32, 8, 128), (16, 2, 64), (3, 3, 128)], ids=lambda h: "%d_%d_%d" % h)
def test_ids_outside_the_pool_are_clamped(heads):
    hq, hkv, d = heads
    b = W.ragged_small(310, "bf16", Hq=hq, Hkv=hkv, d=d, prefix_lens=(700, 37, 1300), new_lens=(40, 70, 1), num_pages=200)
    kb = make(b)
    kb.pool = full_pool(b)
    bad = b.block_table.copy()
    used = [-(-int(p) // 16) for p in b.prefix_lens]
    bad[0, :used[0]:3], bad[1, 1], bad[2, :used[2]:5] = -1, 2 ** 31 - 1, b.num_pages
    bad[2, used[2] - 2] = -2 ** 31
    good = np.clip(bad, 0, b.num_pages - 1).astype(np.int32)
    assert (bad != good).sum() > 30
    dev = DeviceKv8(kb)

    def results(table):
        dev.block_table = to_torch(table)
        outs = [dev.decode(lens=np.minimum(b.prefix_lens, 600)), dev.decode(static=True)]
        for waves in (0, 4, 8, 64):
            binding.set_attn_waves(waves)
            outs.append(dev.prefill())
        binding.set_attn_waves(0)
        k, v = (torch.zeros((sum(b.prefix_lens), hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        binding.read_kv(dev.shape, dev.pool, dev.block_table, [0] * b.B, b.prefix_lens, k, v)
        torch.cuda.synchronize()
        return outs + [k, v]

    try:
        want, got = results(good), results(bad)
    finally:
        binding.set_attn_waves(0)
    for x, y in zip(want, got):
        assert bool(torch.isfinite(x).all()) and torch.equal(x, y)
    # an append to a page that is not there goes to the page the id is clamped to, and nowhere else
    table = b.block_table.copy()
    free = sorted(set(range(b.num_pages)) - set(table.reshape(-1).tolist()))
    swap = {0: free[0], b.num_pages - 1: free[1]}                                  # (the two ends belong to no request)
    table = np.vectorize(lambda p: swap.get(int(p), int(p)))(table).astype(np.int32)
    clamped = table.copy()
    table[0, (700 + 16) // 16], clamped[0, (700 + 16) // 16] = -5, 0
    table[1, (37 + 16) // 16], clamped[1, (37 + 16) // 16] = b.num_pages + 9, b.num_pages - 1
    pools = []
    for t in (clamped, table):
        dev.pool = torch.from_numpy(kb.pool.copy()).cuda()
        dev.block_table = to_torch(t)
        dev.append()
        torch.cuda.synchronize()
        pools.append(dev.pool)
    assert torch.equal(*pools) and bool((pools[0][0] != torch.from_numpy(kb.pool[0]).cuda()).any())


def test_append_beside_a_prefill_of_the_same_pages():
    """Prefixes that end inside a page: the append fills the rest of it, and its scales' line, while the prefill reads the rows before."""
    b = W.ragged_small(311, "bf16", Hq=32, Hkv=8, d=128, prefix_lens=(4097, 999, 15, 2001), new_lens=(300, 37, 600, 5), num_pages=600)
    kb = make(b)
    dev = DeviceKv8(kb)
    alone = dev.prefill()
    after = K8.append_kv(b.k_new, b.v_new, kb.pool, b.block_table, b.prefix_lens, b.new_lens)
    sides = [torch.cuda.Stream() for _ in range(2)]
    for i in range(5):
        dev.pool.copy_(torch.from_numpy(kb.pool).cuda())
        torch.cuda.synchronize()
        out = torch.full_like(dev.q, 7.0)
        torch.cuda.synchronize()
        dev.append(sides[0])
        if i == 4:
            torch.cuda.synchronize()                                             # (once behind it)
        binding.prefix_prefill(dev.shape, dev.q, dev.k_new, dev.v_new, dev.pool, dev.block_table, b.prefix_lens, b.new_lens, out, sides[1])
        torch.cuda.synchronize()
        assert torch.equal(out, alone)
        assert np.array_equal(dev.pool.cpu().numpy(), after)
