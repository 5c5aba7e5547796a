"""The 8-bit pool on the GPU: rows quantised on their way in and read back, bit for bit against the CPU reference; attention over it against
the fp64 oracle on the values that the pool stands for."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import kv8_oracle as K8                                              # noqa: E402
from paper_2605_06472_amd import binding, workloads as W                         # noqa: E402
from tests.gpu_util import DeviceBatch, assert_close, to_numpy, to_torch    # noqa: E402
from tests.kv8_util import DeviceKv8, f64, make                                  # noqa: E402

HEADS = [(8, 2, 128), (4, 4, 64), (4, 2, 64), (16, 2, 64), (16, 1, 64), (32, 2, 128), (32, 8, 128), (3, 3, 128), (8, 8, 128), (16, 2, 128)]
IDS = ["%d_%d_%d" % h for h in HEADS]


def small(seed, heads, **kw):
    hq, hkv, d = heads
    return W.ragged_small(seed, "bf16", Hq=hq, Hkv=hkv, d=d, **kw)


# ---- rows in and out ------------------------------------------------------------------------------------------
def _append(b, before):
    pool = torch.from_numpy(before.copy()).cuda()
    shape = binding.make_shape(b.B, b.Hq, b.Hkv, b.d, b.P, b.num_pages, b.max_pages, "bf16_kv8")
    table = to_torch(b.block_table)
    binding.append_kv(shape, to_torch(b.k_new), to_torch(b.v_new), pool, table, b.prefix_lens, b.new_lens)
    torch.cuda.synchronize()
    return shape, table, pool


@pytest.mark.parametrize("heads", HEADS, ids=IDS)
def test_append_and_read_are_bit_exact(heads):
    b = small(210 + heads[0], heads, prefix_lens=(0, 5, 16, 37, 130, 15), new_lens=(1, 3, 70, 0, 129, 1))
    before = np.full((b.num_pages, K8.page_bytes(b.Hkv, b.d)), 0xA5, np.uint8)
    shape, table, pool = _append(b, before)
    want = K8.append_kv(b.k_new, b.v_new, before, b.block_table, b.prefix_lens, b.new_lens)
    assert np.array_equal(pool.cpu().numpy(), want)          # every byte, those that nothing writes among them
    k, v = (torch.full((b.N + 2, b.Hkv, b.d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.read_kv(shape, pool, table, b.prefix_lens, b.new_lens, k[1:], v[1:])
    torch.cuda.synchronize()
    wk, wv = K8.read_kv(want, b.Hkv, b.d, b.block_table, b.prefix_lens, b.new_lens)
    assert np.array_equal(to_numpy(k[1:-1]), wk) and np.array_equal(to_numpy(v[1:-1]), wv)
    assert all(bool((x[[0, -1]] == 7).all()) for x in (k, v))


def test_append_of_every_kind_of_row():
    """All 65536 bf16 patterns, mixed rows of zeros, subnormals, infinities, NaN and the largest numbers, at both widths."""
    for d in (64, 128):
        every = np.arange(65536, dtype=np.uint16).reshape(-1, d)                  # rows of one magnitude
        rng = np.random.default_rng(3)
        mixed = rng.permutation(65536).astype(np.uint16).reshape(-1, d)           # ... of all at once
        finite = np.where((every & 0x7f80) == 0x7f80, np.uint16(0), every)
        near = W.f32_to_bf16_bits(rng.standard_normal((512, d)).astype(np.float32))
        zero = np.zeros((2, d), np.uint16)
        zero[1] = 0x8000
        rows = np.concatenate([every, mixed, finite, near, zero])
        n = len(rows) // 2
        b = W.ragged_small(33, "bf16", Hq=1, Hkv=1, d=d, prefix_lens=(3,), new_lens=(n,), num_pages=n // 16 + 4)
        b.k_new, b.v_new = rows[:n].reshape(n, 1, d).copy(), rows[n:2 * n].reshape(n, 1, d).copy()
        before = np.zeros((b.num_pages, K8.page_bytes(1, d)), np.uint8)
        shape, table, pool = _append(b, before)
        assert np.array_equal(pool.cpu().numpy(), K8.append_kv(b.k_new, b.v_new, before, b.block_table, b.prefix_lens, b.new_lens))
        k, v = (torch.zeros((n, 1, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        binding.read_kv(shape, pool, table, b.prefix_lens, b.new_lens, k, v)
        wk, wv = K8.read_kv(pool.cpu().numpy(), 1, d, b.block_table, b.prefix_lens, b.new_lens)
        for got, want in ((k, wk), (v, wv)):
            assert np.array_equal(f64(got), W.to_f64(want), equal_nan=True)


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 2, 128)), ("bf16", (4, 4, 64)), ("f32", (6, 3, 64)), ("f32", (2, 1, 128))])
def test_read_of_plain_pools_is_a_copy(dtype, heads):
    hq, hkv, d = heads
    b = W.ragged_small(220, dtype, Hq=hq, Hkv=hkv, d=d)
    db = DeviceBatch(b)
    db.append()
    k, v = torch.zeros_like(db.k_new), torch.zeros_like(db.v_new)
    binding.read_kv(db.shape, db.kv_pool, db.block_table, b.prefix_lens, b.new_lens, k, v)
    torch.cuda.synchronize()
    assert torch.equal(k, db.k_new) and torch.equal(v, db.v_new)
    # a stretch of each prefix, from anywhere
    first, num = np.array([0, 2, 0, 20, 15], np.int32), np.array([0, 3, 16, 17, 115], np.int32)
    k, v = (torch.zeros((int(num.sum()), hkv, d), dtype=db.q.dtype, device="cuda") for _ in range(2))
    binding.read_kv(db.shape, db.kv_pool, db.block_table, first, num, k, v)
    pos = [(r, f + i) for r, (f, n) in enumerate(zip(first, num)) for i in range(n)]
    want = np.stack([b.kv_pool[b.block_table[r, t // 16], :, :, t % 16] for r, t in pos])
    torch.cuda.synchronize()
    assert np.array_equal(to_numpy(k), want[:, 0]) and np.array_equal(to_numpy(v), want[:, 1])


def test_offsets_past_32_bits():
    """Pages behind the first 4 GiB of a pool."""
    hkv, d, pages = 8, 128, 140000                           # 33024 bytes a page
    b = W.ragged_small(221, "bf16", Hq=32, Hkv=hkv, d=d, prefix_lens=(33, 300), new_lens=(40, 5), num_pages=64)
    b.block_table = (b.block_table + pages - 64).astype(np.int32)
    shape = binding.make_shape(b.B, 32, hkv, d, 16, pages, b.max_pages, "bf16_kv8")
    pool = torch.zeros((pages, K8.page_bytes(hkv, d)), dtype=torch.uint8, device="cuda")
    tail = np.zeros((64, pool.shape[1]), np.uint8)
    codes, scales = K8.quantise(b.kv_pool)
    K8.codes_of(tail, hkv, d)[:], K8.scales_of(tail, hkv, d)[:] = codes, np.moveaxis(scales, 1, -1)
    pool[-64:] = torch.from_numpy(tail).cuda()
    q, k, v, table = (to_torch(a) for a in (b.q, b.k_new, b.v_new, b.block_table))
    out = torch.zeros_like(q)
    binding.prefix_prefill(shape, q, k, v, pool, table, b.prefix_lens, b.new_lens, out)
    binding.append_kv(shape, k, v, pool, table, b.prefix_lens, b.new_lens)
    one = torch.zeros_like(q[:2])
    binding.paged_decode(shape, q[:2], pool, table, b.prefix_lens, one)
    torch.cuda.synchronize()
    low = (b.block_table - (pages - 64)).astype(np.int32)
    import oracle
    vals = K8.values(tail, hkv, d)
    assert_close(f64(out), oracle.prefill(b.q, b.k_new, b.v_new, vals, low, b.prefix_lens, b.new_lens), "bf16", "prefill")
    assert_close(f64(one), oracle.decode(b.q[:2], vals, low, b.prefix_lens), "bf16", "decode")
    assert np.array_equal(pool[-64:].cpu().numpy(), K8.append_kv(b.k_new, b.v_new, tail, low, b.prefix_lens, b.new_lens))
    assert not bool(pool[:-64].any())


# ---- decode ------------------------------------------------------------------------------------------------
CONTEXTS = (1, 15, 16, 17, 64, 130, 1000, 0, 4097, 31, 333)


def decode_close(got, want, b, values, lens, what):
    """The rounding of the result to bf16 (half a step: 2^-8 of it), and fp32 arithmetic: scores that are sums of d products, off by
    (d + 8) 2^-24 of the largest score there is, move weights by as much, sums over the context by L 2^-24; both move a result by
    at most twice that times the largest |v|."""
    v = np.abs(np.nan_to_num(W.to_f64(values)))
    top = np.sqrt((W.to_f64(b.q) ** 2).sum(-1).max() * (v[:, 0] ** 2).sum(-1).max() / b.d)
    off = 2 * v[:, 1].max() * 2.0 ** -24 * ((b.d + 8) * top + max(lens))
    err = np.abs(got - want)
    assert np.isfinite(got).all(), what
    assert (err <= 2.0 ** -8 * np.abs(want) + off).all(), "%s: %.3e" % (what, (err - 2.0 ** -8 * np.abs(want)).max())


@pytest.mark.parametrize("heads", HEADS, ids=IDS)
def test_decode_matches_the_oracle(oracle, heads):
    kb = make(small(230 + heads[0], heads, prefix_lens=CONTEXTS, new_lens=(1,) * len(CONTEXTS), num_pages=640))
    d = DeviceKv8(kb)
    want = oracle.decode(kb.b.q, kb.values, kb.b.block_table, kb.b.prefix_lens)
    got = d.decode()
    decode_close(f64(got), want, kb.b, kb.values, CONTEXTS, "decode %s" % (heads,))
    assert not bool(got[CONTEXTS.index(0)].any())
    assert torch.equal(d.decode(static=True), got) and torch.equal(d.decode(), got)
    lens = [max(0, c - 1 - 7 * (i % 3)) for i, c in enumerate(CONTEXTS)]          # inside what the pages hold
    decode_close(f64(d.decode(lens)), oracle.decode(kb.b.q, kb.values, kb.b.block_table, lens), kb.b, kb.values, lens, "shorter")


@pytest.mark.parametrize("heads,batch,ctx", [((32, 8, 128), 300, (1, 90)), ((16, 2, 64), 700, (1, 300)), ((32, 2, 128), 140, (200, 2000)), ((16, 2, 128), 64, (500, 6000)),
                                             ((8, 8, 128), 3, (9000, 12000)), ((4, 4, 64), 1, (20000, 20000))],
                         ids=["many_short", "many_d64", "g16", "g8", "g1", "one_long_d64"])
def test_decode_of_larger_batches(oracle, heads, batch, ctx):
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(ctx[0], ctx[1] + 1, batch)]
    kb = make(small(240 + batch, heads, prefix_lens=lens, new_lens=(1,) * batch, num_pages=sum(-(-(x + 1) // 16) for x in lens) + 8))
    d = DeviceKv8(kb)
    got = d.decode()
    decode_close(f64(got), oracle.decode(kb.b.q, kb.values, kb.b.block_table, lens), kb.b, kb.values, lens, "decode")
    assert torch.equal(d.decode(), got)


def test_decode_slices_of_more_pages_than_a_wave_holds_ids_for(oracle):
    """A call so large that its contexts stay in slices of a thousand pages: many requests over the same pages, in two orders."""
    hkv, d, pages, ctx, batch = 8, 128, 1000, 15997, 280
    b = small(251, (32, 8, 128), prefix_lens=(ctx, ctx), new_lens=(1, 1), num_pages=2 * pages + 2)
    kb = make(b)
    want = oracle.decode(b.q, kb.values, b.block_table, b.prefix_lens)
    table = to_torch(b.block_table).repeat(batch // 2, 1).contiguous()
    q = to_torch(b.q).repeat(batch // 2, 1, 1).contiguous()
    shape = binding.make_shape(batch, 32, hkv, d, 16, b.num_pages, b.max_pages, "bf16_kv8")
    out = torch.full_like(q, 7.0)
    binding.paged_decode(shape, q, torch.from_numpy(kb.pool).cuda(), table, np.full(batch, ctx, np.int32), out)
    got = f64(out).reshape(batch // 2, 2, 32, d)
    assert (got == got[:1]).all()
    decode_close(got[0], want, b, kb.values, (ctx,), "decode")


def test_decode_over_scales_of_every_size(oracle):
    """Keys and values whose rows lie far apart in magnitude, and a maximum that comes late."""
    b = small(250, (8, 2, 128), prefix_lens=(700, 33, 1200), new_lens=(1,) * 3, num_pages=160)
    x = W.to_f64(b.kv_pool)
    rng = np.random.default_rng(1)
    x[:, 0] *= 2.0 ** rng.integers(-30, 3, x[:, 0].shape[:-1])[..., None]
    x[:, 1] *= 2.0 ** rng.integers(-60, 1, x[:, 1].shape[:-1])[..., None]
    b.kv_pool = W.f32_to_bf16_bits(x.astype(np.float32))
    kb = make(b)
    d = DeviceKv8(kb)
    decode_close(f64(d.decode()), oracle.decode(b.q, kb.values, b.block_table, b.prefix_lens), b, kb.values, b.prefix_lens, "decode")
    prefill_close(f64(d.prefill()), oracle.prefill(b.q, b.k_new, b.v_new, kb.values, b.block_table, b.prefix_lens, b.new_lens), "prefill")


# ---- prefill ----------------------------------------------------------------------------------------------------
PREFILL = {
    "plain": {},
    "tails": dict(prefix_lens=(300, 77, 1000, 0, 64, 16), new_lens=(200, 65, 130, 257, 1, 33), num_pages=200),
    "cut": dict(prefix_lens=(4000, 333, 2047), new_lens=(33, 5, 64), num_pages=440),
    "one_token": dict(prefix_lens=(1, 63, 64, 65, 2000), new_lens=(1,) * 5, num_pages=160),
    "long": dict(prefix_lens=(6500, 7000), new_lens=(300, 70), num_pages=900),
}


# Two roundings to bf16, of the probabilities and of the result, each at most half a step: 2^-8 of the value, and over many values (evenly spread over a step that is 2^-7 to
# 2^-8 of the value) 2^-7 / sqrt(12) / sqrt(2) or less of it as a mean square.  The result's is 1.7e-3 of the norm, that of the probabilities
# as much at most: where few of them count they are a result's error one to one.  Their squares' sum is 2.4e-3; everything else is fp32.
PREFILL_REL = 2.6e-3


def prefill_close(got, want, what):
    assert np.isfinite(got).all(), what
    rel = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert rel <= PREFILL_REL, "%s: %.2e" % (what, rel)
    assert_close(got, want, "bf16", what)


@pytest.mark.parametrize("case", sorted(PREFILL))
@pytest.mark.parametrize("heads", HEADS, ids=IDS)
def test_prefill_matches_the_oracle_in_every_shape(oracle, heads, case):
    """... and has the same bits in every work-group shape, and again."""
    kb = make(small(260 + heads[0], heads, **PREFILL[case]))
    d = DeviceKv8(kb)
    b = kb.b
    want = oracle.prefill(b.q, b.k_new, b.v_new, kb.values, b.block_table, b.prefix_lens, b.new_lens)
    try:
        got = {}
        for waves in (0, 4, 8, 64):
            binding.set_attn_waves(waves)
            got[waves] = d.prefill()
            assert torch.equal(got[waves], d.prefill()), "again, %d waves" % waves
    finally:
        binding.set_attn_waves(0)
    for waves in (0, 4):
        prefill_close(f64(got[waves]), want, "prefill %s, %d waves" % (heads, waves))
    assert torch.equal(got[4], got[8]) and torch.equal(got[4], got[64])


def test_prefill_behind_a_shared_prompt_and_on_scattered_pages(oracle):
    kb = make(small(270, (32, 8, 128), prefix_lens=(0, 40, 500), new_lens=(70, 33, 1), shared_root=1024, num_pages=200))
    d = DeviceKv8(kb)
    b = kb.b
    prefill_close(f64(d.prefill()), oracle.prefill(b.q, b.k_new, b.v_new, kb.values, b.block_table, b.prefix_lens, b.new_lens), "prefill")


def test_peaked_scores_and_masked_keys(oracle):
    """Scores of hundreds, a maximum that comes late, and prefix keys whose scores are -inf or the type's lowest value."""
    for seed, kw in ((272, dict(q_scale=8.0)), (273, dict(q_scale=64.0))):
        kb = make(small(seed, (8, 2, 128), prefix_lens=(700, 33, 2000), new_lens=(40, 20, 3), num_pages=220, **kw))
        d = DeviceKv8(kb)
        b = kb.b
        prefill_close(f64(d.prefill()), oracle.prefill(b.q, b.k_new, b.v_new, kb.values, b.block_table, b.prefix_lens, b.new_lens), "peaked")
    b = small(274, (8, 2, 128), prefix_lens=(300,), new_lens=(20,), num_pages=32)
    k = W.to_f64(b.kv_pool)
    page = b.block_table[0, :10]
    k[page, 0] = -3e38                                       # the first 160 keys: against queries of positive sum -inf, others +inf
    b.kv_pool, b.q = W.f32_to_bf16_bits(k.astype(np.float32)), W.f32_to_bf16_bits(np.abs(W.to_f64(b.q)).astype(np.float32))
    kb = make(b)
    d = DeviceKv8(kb)
    tail = small(274, (8, 2, 128), prefix_lens=(300,), new_lens=(20,), num_pages=32)
    tail.q, tail.kv_pool, tail.block_table, tail.prefix_lens = b.q, b.kv_pool, b.block_table[:, 10:].copy(), np.array([140], np.int32)
    want = oracle.prefill(tail.q, tail.k_new, tail.v_new, kb.values, tail.block_table, tail.prefix_lens, tail.new_lens)
    try:
        for waves in (0, 4, 64):
            binding.set_attn_waves(waves)
            prefill_close(f64(d.prefill()), want, "masked, %d waves" % waves)
    finally:
        binding.set_attn_waves(0)


def test_an_infinity_shows():
    """Infinities and NaN among the keys or values that a row attends to make it NaN, in both attentions; other requests are untouched."""
    b = small(271, (8, 2, 128), prefix_lens=(40, 700, 40), new_lens=(5, 5, 5), num_pages=160)
    clean = DeviceKv8(make(b))
    want = clean.prefill()
    for kv, bits in ((0, 0x7f80), (1, 0xff80), (0, 0x7fc0), (1, 0x7fc1)):
        b.kv_pool[b.block_table[1, 3], kv, 1, 2, 77] = bits
        d = DeviceKv8(make(b))
        got = d.prefill()
        b.kv_pool[b.block_table[1, 3], kv, 1, 2, 77] = 0
        rows = got[5:10, 4:].float()
        assert bool(torch.isnan(rows if kv == 0 else rows[..., 77]).all())
        assert bool(torch.isfinite(got[5:10, :4]).all())
        assert torch.equal(got[:5], want[:5]) and torch.equal(got[10:], want[10:])
        one = torch.zeros_like(d.q[:3])
        binding.paged_decode(d.shape, d.q[:3], d.pool, d.block_table, b.prefix_lens, one)
        assert bool(torch.isnan(one[1, 4:] if kv == 0 else one[1, 4:, 77]).all()) and bool(torch.isfinite(one[[0, 2]]).all())
        assert bool(torch.isfinite(one[1, :4]).all())


def test_rows_of_q_two_gib_apart(oracle):
    """So many heads that tokens of a wave lie 2 GiB apart in q: the form that reaches them."""
    heads, d, n, p = 262144, 128, 33, 20
    g = torch.Generator(device="cuda").manual_seed(9)
    rnd = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(0, 0.5, generator=g)      # noqa: E731
    shape = binding.make_shape(1, heads, heads, d, 16, 4, 4, "bf16_kv8")
    pool = torch.zeros((4, K8.page_bytes(heads, d)), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32, device="cuda")
    zero, pre, new = np.array([0], np.int32), np.array([p], np.int32), np.array([n], np.int32)
    k0, v0 = rnd(p, heads, d), rnd(p, heads, d)
    binding.append_kv(shape, k0, v0, pool, table, zero, pre)
    k, v = torch.zeros_like(k0), torch.zeros_like(v0)
    binding.read_kv(shape, pool, table, zero, pre, k, v)
    q, k_new, v_new = rnd(n, heads, d), rnd(n, heads, d), rnd(n, heads, d)
    out = torch.full_like(q, 7.0)
    binding.prefix_prefill(shape, q, k_new, v_new, pool, table, pre, new, out)
    torch.cuda.synchronize()
    for h in (0, 1, heads // 2 + 3, heads - 1):
        assert (k[:, h].float() - k0[:, h].float()).abs().max() <= 2.0 ** -4 * k0[:, h].float().abs().max()
        keys, vals = (torch.cat((a[:, h], c[:, h])).double() for a, c in ((k, k_new), (v, v_new)))
        s = q[:, h].double() @ keys.T / d ** 0.5
        s.masked_fill_(torch.arange(p + n, device="cuda") > p + torch.arange(n, device="cuda")[:, None], -float("inf"))
        prefill_close(f64(out[:, h]), (torch.softmax(s, -1) @ vals).cpu().numpy(), "head %d" % h)


# ---- as a server uses them ------------------------------------------------------------------------------------------
def test_a_conversation_with_its_cache_in_8_bits(oracle):
    """Prefill, append, decode steps that append as they go, pages out to the host and back into another pool, read, and a next turn
    over what was swapped: every step against the reference's pool."""
    b = small(280, (32, 8, 128), prefix_lens=(0, 37, 333), new_lens=(150, 70, 33), num_pages=128)
    steps = 5
    kb = make(b)
    d = DeviceKv8(kb)
    width = b.max_pages + 2
    table = np.zeros((3, width), np.int32)
    free = [p for p in range(b.num_pages) if p not in set(b.block_table.reshape(-1).tolist())]
    for r in range(3):
        used = -(-(int(b.prefix_lens[r]) + int(b.new_lens[r])) // 16)
        table[r, :used] = b.block_table[r, :used]
        table[r, used:used + 1] = free[r]
    b.block_table = table
    shape = binding.make_shape(3, b.Hq, b.Hkv, b.d, 16, b.num_pages, width, "bf16_kv8")
    tab, pool, host = to_torch(table), d.pool, kb.pool
    out = torch.zeros_like(d.q)
    binding.prefix_prefill(shape, d.q, d.k_new, d.v_new, pool, tab, b.prefix_lens, b.new_lens, out)
    binding.append_kv(shape, d.k_new, d.v_new, pool, tab, b.prefix_lens, b.new_lens)
    assert_close(f64(out), oracle.prefill(b.q, b.k_new, b.v_new, K8.values(host, 8, 128), table, b.prefix_lens, b.new_lens), "bf16", "prefill")
    host = K8.append_kv(b.k_new, b.v_new, host, table, b.prefix_lens, b.new_lens)
    lens = (b.prefix_lens + b.new_lens).astype(np.int32)
    ones = np.ones(3, np.int32)
    for step in range(steps):
        q, k, v = (W.normal_tensor(900 + step, i, (3, h, 128), 2 ** -0.5, "bf16") for i, h in ((0, 32), (1, 8), (2, 8)))
        binding.append_kv(shape, to_torch(k), to_torch(v), pool, tab, lens, ones)
        host = K8.append_kv(k, v, host, table, lens, ones)
        lens = lens + 1
        got = torch.zeros((3, 32, 128), dtype=torch.bfloat16, device="cuda")
        binding.paged_decode(shape, to_torch(q), pool, tab, lens, got)
        vals = K8.values(host, 8, 128)
        assert_close(f64(got), oracle.decode(q, vals, table, lens), "bf16", "decode step %d" % step)
    assert np.array_equal(pool.cpu().numpy(), host)
    # the whole cache through the host tier into another pool, at other pages
    rng = np.random.default_rng(5)
    ids = np.unique(table).astype(np.int32)
    staging = torch.zeros((len(ids), pool.shape[1]), dtype=torch.uint8).pin_memory()
    binding.swap_out_pages(shape, pool, ids, staging)
    torch.cuda.synchronize()
    to = rng.permutation(b.num_pages)[:len(ids)].astype(np.int32)
    other = torch.full_like(pool, 0xFF)
    binding.swap_in_pages(shape, staging, to, other)
    moved = to[np.searchsorted(ids, table)].astype(np.int32)
    tab2 = to_torch(moved)
    k, v = (torch.zeros((int(lens.sum()), 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.read_kv(shape, other, tab2, np.zeros(3, np.int32), lens, k, v)
    wk, wv = K8.read_kv(host, 8, 128, table, np.zeros(3, int), lens)
    torch.cuda.synchronize()
    assert np.array_equal(to_numpy(k), wk) and np.array_equal(to_numpy(v), wv)
    new = np.array([4, 0, 17], np.int32)
    q, k, v = (W.normal_tensor(990, i, (21, h, 128), 2 ** -0.5, "bf16") for i, h in ((0, 32), (1, 8), (2, 8)))
    out = torch.zeros((21, 32, 128), dtype=torch.bfloat16, device="cuda")
    wide = np.concatenate([moved, np.zeros((3, 2), np.int32)], 1)
    shape2 = binding.make_shape(3, 32, 8, 128, 16, b.num_pages, width + 2, "bf16_kv8")
    binding.prefix_prefill(shape2, to_torch(q), to_torch(k), to_torch(v), other, to_torch(wide), lens, new, out)
    wide0 = np.concatenate([table, np.zeros((3, 2), np.int32)], 1)
    assert_close(f64(out), oracle.prefill(q, k, v, K8.values(host, 8, 128), wide0, lens, new), "bf16", "next turn")


def test_calls_on_two_streams(oracle):
    """Two batches at once, a bf16 pool's call between them on the same streams."""
    kbs = [make(small(290 + i, (32, 8, 128), prefix_lens=p, new_lens=n, num_pages=700)) for i, (p, n) in
           enumerate((((700, 4097, 33), (64, 40, 1)), ((1500, 9, 2500), (1, 130, 20))))]
    ds = [DeviceKv8(kb) for kb in kbs]
    want = [d.prefill() for d in ds]
    plain = [d.prefill(plain=True) for d in ds]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for k in range(4):
        for i in (0, 1):
            got.append((i, ds[i].prefill(stream=streams[(i + k) % 2])))
            got.append((i, ds[1 - i].prefill(plain=True, stream=streams[(i + k) % 2])))
    torch.cuda.synchronize()
    for n, (i, out) in enumerate(got):
        assert torch.equal(out, want[i] if n % 2 == 0 else plain[1 - i])


def test_static_decode_in_a_graph():
    """Captured, and replayed with eager work between the replays: over what the pool holds then."""
    kb = make(small(300, (16, 2, 64), prefix_lens=(4097, 17, 0, 600), new_lens=(1,) * 4, num_pages=330))
    d = DeviceKv8(kb)
    b = kb.b
    out = torch.zeros_like(d.q)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    d.decode(static=True)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        binding.paged_decode_static(d.shape, d.q, d.pool, d.block_table, b.prefix_lens, out, side)
    for k in range(3):
        d.q.mul_(-1.0 if k % 2 else 0.5)
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, d.decode())
    with pytest.raises(binding.PbkvError) as e:
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
            binding.read_kv(d.shape, d.pool, d.block_table, b.prefix_lens, b.new_lens, d.k_new, d.v_new, side)
    assert e.value.code == -6
