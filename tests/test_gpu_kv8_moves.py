"""Pages of an 8-bit pool through the host tier, more of them than a launch of the swaps has work-groups for; rows read back from plain pools behind
their first 4 GiB."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2605_06472_amd import binding                                         # noqa: E402


@pytest.mark.parametrize("hkv,d", [(8, 128), (2, 64), (1, 64), (5, 128)])
def test_swaps_of_many_pages(hkv, d):
    pages, moved = 700, 333
    shape = binding.make_shape(1, hkv, hkv, d, 16, pages, 1, "bf16_kv8")
    nbytes = binding.page_bytes(shape)
    g = torch.Generator(device="cuda").manual_seed(hkv)
    pool = torch.randint(0, 256, (pages, nbytes), dtype=torch.uint8, device="cuda", generator=g)
    before = pool.clone()
    rng = np.random.default_rng(hkv)
    out_ids = rng.integers(0, pages, moved).astype(np.int32)                      # some of them twice
    host = torch.empty((moved, nbytes), dtype=torch.uint8, pin_memory=True)
    binding.swap_out_pages(shape, pool, out_ids, host)
    torch.cuda.synchronize()
    assert torch.equal(pool, before)
    assert torch.equal(host, before.cpu()[torch.from_numpy(out_ids).long()])
    in_ids = rng.permutation(pages)[:moved].astype(np.int32)
    binding.swap_in_pages(shape, host, in_ids, pool)
    torch.cuda.synchronize()
    want = before.clone()
    want[torch.from_numpy(in_ids).long().cuda()] = host.cuda()
    assert torch.equal(pool, want)


@pytest.mark.parametrize("dtype,hkv,d", [("bf16", 8, 128), ("f32", 4, 128), ("f32", 16, 64)])
def test_reads_past_32_bits(dtype, hkv, d):
    shape = binding.make_shape(2, hkv, hkv, d, 16, 70000, 25, dtype)
    assert (70000 - 60) * binding.page_bytes(shape) > 1 << 32
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    pool = torch.zeros((70000, 2, hkv, 16, d), dtype=t, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    pool[-60:] = torch.empty((60, 2, hkv, 16, d), dtype=t, device="cuda").normal_(generator=g)
    table = torch.randperm(60, generator=torch.Generator().manual_seed(1))[:50].reshape(2, 25).to(torch.int32) + 70000 - 60
    first, num = np.array([3, 0], np.int32), np.array([390, 17], np.int32)
    k, v = (torch.full((407, hkv, d), 7.0, dtype=t, device="cuda") for _ in range(2))
    binding.read_kv(shape, pool, table.cuda(), first, num, k, v)
    torch.cuda.synchronize()
    at = [(int(table[r, (f + i) // 16]), (int(f) + i) % 16) for r, (f, n) in enumerate(zip(first, num)) for i in range(n)]
    page, slot = (torch.tensor(x, device="cuda") for x in zip(*at))
    want = pool[page, :, :, slot]
    assert torch.equal(k, want[:, 0]) and torch.equal(v, want[:, 1])
