"""Performance cases of the 8-bit KV cache: what a serving program has the library do with it, through the Python binding.

Four kinds of pass over a paged pool whose K and V rows are held in e4m3 with a power-of-two scale per row (dtype "bf16_kv8"):

  write      the K/V of a batch's new tokens are quantised into the pool (``append_kv``), and the same tokens read back (``read_kv``),
             as where a request's cache moves on to another pool
  read       a stretch of every request's cache comes back as packed bf16 rows (``read_kv``)
  decode     one query row per request over its whole context (``paged_decode``, or ``paged_decode_static``)
  prefill    the new tokens of a batch attend to their cached prefix pages and causally to themselves (``prefix_prefill``)

A page of the pool is one run of bytes: the codes [K, V][KV head][slot of 16][d], then the scale bytes [KV head][slot][K, V]
(byte b stands for 2 ** (b - 127)), then nothing up to a multiple of 128 bytes.

The lengths of a case follow from its own fields (``lens_seed`` among them); values and page placement follow from the seed that
``prepare`` is given.  Q, K and V are N(0, 1/2) as the synthetic workloads of this repository draw them, with one K channel in 32 eight times
as wide, as the K of language models has it.  Slots of the pool that hold no token are filled with NaN codes.
"""
import math
import random

import numpy as np
import torch

own = False      # True: the library's calls; False: the same in elementary operations

PAGE = 16
BENCH_HEADS = (32, 8, 128)
# (query heads, KV heads, head width): every head ratio and both widths
HEADS = (BENCH_HEADS, (8, 2, 128), (8, 2, 64), (4, 2, 128), (16, 2, 128), (16, 2, 64), (16, 1, 64), (32, 2, 128), (4, 4, 64), (8, 8, 128))
MAX_FLOPS = 2.4e12      # a drawn prefill does no more arithmetic than the largest listed one
MAX_BYTES = 1.2e9       # ... and a drawn decode reads no more than the largest listed one
MAX_COPY_BYTES = 4.2e8  # ... nor a drawn write or read
MAX_SCORES = 5e9        # what the plain form holds at once, padded to the longest request


def _case(name, kind, batch, prefix, new, heads=BENCH_HEADS, root=0, static=False, lens_seed=1):
    return {"name": name, "kind": kind, "batch": batch, "hq": heads[0], "hkv": heads[1], "d": heads[2], "root": root, "static": static,
            "prefix_min": prefix[0], "prefix_max": prefix[1], "new_min": new[0], "new_max": new[1], "lens_seed": lens_seed}


def listed():
    return [
        # a decode step of 64 requests: one token each, at any place of its page
        _case("write_step", "write", 64, (1023, 16383), (1, 1)),
        # cold prompts of a narrow-head model, ragged, some behind a few tokens of another page
        _case("write_ragged_d64", "write", 6, (0, 40), (100, 2000), heads=(16, 2, 64)),
        # one long document, prefilled behind a greeting
        _case("write_document", "write", 1, (5, 5), (32768, 32768)),
        # a conversation's cache on its way to another pool
        _case("read_history", "read", 1, (3, 3), (12001, 12001)),
        # the caches of 16 requests of a narrow-head model
        _case("read_batch_d64", "read", 16, (0, 16), (1, 4096), heads=(16, 2, 64)),
        # one user, one short conversation: the smallest call a server makes, once per layer and token
        _case("decode_one", "decode", 1, (1003, 1003), (0, 0)),
        # the decode batch prefetch transfers hide behind: 64 requests, contexts U{1024..16384}
        _case("decode_batch", "decode", 64, (1024, 16384), (0, 0)),
        # a narrow-head model in a serving loop that may not allocate, ragged short contexts
        _case("decode_static_d64", "decode", 24, (17, 4097), (0, 0), heads=(16, 2, 64), static=True),
        # an agent's next turn: a tool result of a few dozen tokens on a long private history
        _case("prefill_turn", "prefill", 1, (12001, 12001), (37, 37)),
        # four requests behind one shared 2048-token system prompt, 512 new tokens each
        _case("prefill_shared_prompt", "prefill", 4, (0, 0), (512, 512), root=2048),
        # two long accumulated histories, 2048 new tokens each
        _case("prefill_long_history", "prefill", 2, (32768, 32768), (2048, 2048)),
        # requests of a narrow-head model, ragged, some with next to nothing cached
        _case("prefill_ragged_d64", "prefill", 6, (0, 1500), (100, 2000), heads=(16, 2, 64)),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        case = _draw(rng)
        del case["name"]
        w = work(case)
        prefix, new = _lens(case)
        longest = case["root"] + max(prefix) + max(new)
        rows = max(1, max(new)) if case["kind"] == "prefill" else 1
        padded = case["batch"] * longest * max(case["hq"] * rows, 2 * case["hkv"] * case["d"])
        most = MAX_BYTES if case["kind"] in ("decode", "prefill") else MAX_COPY_BYTES
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= most and padded <= MAX_SCORES:
            return case


def _draw(rng):
    heads = BENCH_HEADS if rng.random() < 0.5 else rng.choice(HEADS)
    kind, lens_seed = rng.choice(("write", "read", "decode", "decode", "prefill", "prefill")), rng.randrange(1 << 20)
    if kind == "decode":
        hi, batch = _log_int(rng, 40, 32768), _log_int(rng, 1, 128)
        static = rng.random() < 0.4 and batch <= 64 and batch * hi <= 100000      # inside that entry point's limits
        return _case("", kind, batch, (max(1, hi // rng.choice((1, 2, 16))), hi), (0, 0), heads, 0, static, lens_seed)
    hi, new = _log_int(rng, 16, 32768), _log_int(rng, 1, 2048 if kind == "prefill" else 32768)
    lo = rng.choice((0, hi // 4, hi))
    if rng.random() < 0.1:
        hi = lo = 0
    root = PAGE * _log_int(rng, 1, 128) if kind == "prefill" and rng.random() < 0.3 else 0
    return _case("", kind, _log_int(rng, 1, 32), (lo, hi), (max(1, new // rng.choice((1, 1, 8))), new), heads, root, False, lens_seed)


def _lens(case):
    """Private prefix tokens (behind the shared root) and new tokens of every request."""
    rng = random.Random(case["lens_seed"])
    pairs = [(rng.randint(case["prefix_min"], case["prefix_max"]), rng.randint(case["new_min"], case["new_max"])) for _ in range(case["batch"])]
    return [p for p, _ in pairs], [n for _, n in pairs]


# ---- what one pass cannot do without ------------------------------------------------------------------
def work(case):
    hq, hkv, d, root = case["hq"], case["hkv"], case["d"], case["root"]
    prefix, new = _lens(case)
    code, plain = 2 * hkv * (d + 1), 2 * hkv * d * 2      # bytes of a token's K and V in the pool, and in bf16
    if case["kind"] == "write":                           # bf16 rows in, codes out; codes in, bf16 rows out
        return {"bytes": float(sum(new) * 2 * (plain + code)), "flops": 0.0}
    if case["kind"] == "read":
        return {"bytes": float(sum(new) * (plain + code)), "flops": 0.0}
    if case["kind"] == "decode":
        return {"bytes": float(sum(prefix) * code + case["batch"] * 2 * hq * d * 2), "flops": 4.0 * d * hq * sum(prefix)}
    flops = sum(4 * d * hq * (n * (root + p) + n * (n + 1) // 2) for p, n in zip(prefix, new))
    return {"bytes": float((root + sum(prefix)) * code + sum(new) * (plain + 2 * hq * d * 2)), "flops": float(flops)}


# ---- the pool's format -----------------------------------------------------------------------------------
def _page_bytes(hkv, d):
    return -(-(2 * hkv * PAGE * (d + 1)) // 128) * 128


def _codes(pool, hkv, d):
    """[page][K, V][KV head][slot][d], as bytes."""
    return pool[:, :2 * hkv * PAGE * d].view(pool.shape[0], 2, hkv, PAGE, d)


def _scale_bytes(pool, hkv, d):
    """[page][KV head][slot][K, V]"""
    return pool[:, 2 * hkv * PAGE * d:2 * hkv * PAGE * (d + 1)].view(pool.shape[0], hkv, PAGE, 2)


def _power(exponent):
    """2 ** exponent in fp32, exactly."""
    return ((exponent.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """Rows of bf16 -> e4m3 codes and scale bytes: the smallest power of two with which the row's largest finite value is at most 448."""
    x = x.float()
    fine = torch.isfinite(x)
    largest = torch.where(fine, x.abs(), 0.0).amax(-1)
    mantissa, exponent = torch.frexp(largest)             # in [1/2, 1), and 448 is 7/8 of 512
    exponent = torch.where(largest > 0, exponent - 9 + (mantissa > 0.875), -111).clamp(-111, 119).int()
    scaled = (x * _power(-exponent)[..., None]).clamp(-448.0, 448.0)
    codes = torch.where(fine, scaled, math.nan).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), (exponent + 127).to(torch.uint8)


def _values(codes, scales):
    """What codes [..., d] with scale bytes [...] stand for, in fp32."""
    return codes.view(torch.float8_e4m3fn).float() * _power(scales.int() - 127)[..., None]


# ---- what a program has in hand before the call --------------------------------------------------------
def _normal(g, shape, spread=None):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) * 2 ** -0.5
    return x if spread is None else x * spread


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    host = np.random.default_rng(seed)
    hq, hkv, d, root, batch = case["hq"], case["hkv"], case["d"], case["root"], case["batch"]
    private, new = _lens(case)
    # the shared root's pages, then every request's own, on scattered pages of a pool that holds a third more than is used
    used = root // PAGE
    rows = []
    for p, n in zip(private, new):
        mine = -(-(p + n) // PAGE)
        rows.append(list(range(root // PAGE)) + list(range(used, used + mine)))
        used += mine
    pool_pages, width = used + used // 3 + 3, max(1, max(map(len, rows)))
    place = host.permutation(pool_pages).astype(np.int32)
    table = np.zeros((batch, width), np.int32)
    for r, row in enumerate(rows):
        table[r, :len(row)] = place[np.asarray(row, np.int64)]
    prefix, new = np.array(private, np.int32) + root, np.array(new, np.int32)
    total = int(new.sum())
    # the pool: every slot that holds a token (of a request to be read or attended to) its codes, all others NaN
    pool = torch.full((pool_pages, _page_bytes(hkv, d)), 0xFF, dtype=torch.uint8, device="cuda")
    wide = torch.where(torch.arange(d, device="cuda") % 32 == 5, 8.0, 1.0).to(torch.bfloat16)
    held = prefix + new if case["kind"] in ("read", "write") else prefix
    slots = np.zeros((pool_pages, PAGE), bool)
    for r in range(batch):
        whole, rest = divmod(int(held[r]), PAGE)
        slots[table[r, :whole]] = True
        if rest:
            slots[table[r, whole], :rest] = True
    live = torch.from_numpy(slots).cuda()
    for kv in range(2):
        codes, scales = _quantise(_normal(g, (pool_pages, hkv, PAGE, d), wide if kv == 0 else None))
        _codes(pool, hkv, d)[:, kv] = torch.where(live[:, None, :, None], codes, 0xFF)
        _scale_bytes(pool, hkv, d)[..., kv] = torch.where(live[:, None, :], scales, 0xFF)
    state = {"kind": case["kind"], "static": case["static"], "hq": hq, "hkv": hkv, "d": d, "pool": pool, "table": torch.from_numpy(table).cuda(),
             "prefix_lens": prefix, "new_lens": new, "sizes": (batch, hq, hkv, d, PAGE, pool_pages, width)}
    # where every new token stands: its request, its number there, its position in the request's context
    request = np.repeat(np.arange(batch), new)
    number = np.arange(total) - np.repeat(np.cumsum(new) - new, new)
    for name, a in (("request", request), ("number", number), ("position", number + prefix[request]), ("context", prefix)):
        state[name] = torch.from_numpy(a.astype(np.int64)).cuda()
    if case["kind"] in ("decode", "prefill"):
        state["q"] = _normal(g, (batch if case["kind"] == "decode" else total, hq, d))
        state["out"] = torch.zeros_like(state["q"])
    if case["kind"] in ("write", "prefill"):
        state["k_new"], state["v_new"] = _normal(g, (total, hkv, d), wide), _normal(g, (total, hkv, d))
    if case["kind"] in ("write", "read"):
        state["k"], state["v"] = (torch.zeros((total, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return state


# ---- one pass ------------------------------------------------------------------------------------------
def run(state):
    if own:
        return _run_own(state)
    s, hkv, d = state, state["hkv"], state["d"]
    codes, scales = _codes(s["pool"], hkv, d), _scale_bytes(s["pool"], hkv, d)
    if s["kind"] in ("write", "read"):
        page, slot = s["table"][s["request"], s["position"] // PAGE].long(), s["position"] % PAGE
        if s["kind"] == "write":
            (kc, ks), (vc, vs) = _quantise(s["k_new"]), _quantise(s["v_new"])
            codes[page, 0, :, slot], codes[page, 1, :, slot] = kc, vc
            scales[page, :, slot] = torch.stack((ks, vs), -1)
        row_scales = scales[page, :, slot]
        return {"k": _values(codes[page, 0, :, slot], row_scales[..., 0]).bfloat16(), "v": _values(codes[page, 1, :, slot], row_scales[..., 1]).bfloat16()}
    # attention: whole contexts gathered by pages and padded to the longest, q [request][KV head][row, query head of the group][d]
    context, batch, group = s["context"], s["table"].shape[0], s["hq"] // hkv
    pages = s["table"][:, :-(-int(s["prefix_lens"].max()) // PAGE)].long()
    longest = pages.shape[1] * PAGE
    row_scales = scales[pages].permute(4, 0, 2, 1, 3)
    k, v = (_values(codes[pages, kv].permute(0, 2, 1, 3, 4), row_scales[kv]).reshape(batch, hkv, longest, d) for kv in range(2))
    seen = torch.arange(longest, device="cuda") < context[:, None]
    if s["kind"] == "decode":
        q, new = s["q"].float()[:, None], None
    else:
        new = int(s["new_lens"].max())
        q = torch.zeros((batch, new, s["hq"], d), device="cuda")
        k_new, v_new = (torch.zeros((batch, new, hkv, d), device="cuda") for _ in range(2))
        q[s["request"], s["number"]], k_new[s["request"], s["number"]], v_new[s["request"], s["number"]] = s["q"].float(), s["k_new"].float(), s["v_new"].float()
        k, v = torch.cat((k, k_new.transpose(1, 2)), 2), torch.cat((v, v_new.transpose(1, 2)), 2)
    tokens = q.shape[1]
    q = q.view(batch, tokens, hkv, group, d).permute(0, 2, 1, 3, 4)
    mask = seen[:, None].expand(batch, tokens, longest)
    if new is not None:
        causal = torch.arange(new, device="cuda") <= torch.arange(new, device="cuda")[:, None]
        mask = torch.cat((mask, causal.expand(batch, new, new)), 2)
    v = torch.where(mask[:, -1, None, :, None], v, 0.0)
    scores = torch.matmul(q.reshape(batch, hkv, tokens * group, d), k.transpose(2, 3).contiguous()).view(batch, hkv, tokens, group, -1)
    scores = torch.where(mask[:, None, :, None], scores * d ** -0.5, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-3e38) if scores.shape[-1] else scores.new_zeros(scores.shape[:-1] + (1,))
    weights = torch.exp(scores - top)
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights.view(batch, hkv, tokens * group, -1), v).view(batch, hkv, tokens, group, d)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 2, 1, 3, 4).reshape(batch, tokens, s["hq"], d).bfloat16()
    s["out"] = out[:, 0] if new is None else out[s["request"], s["number"]]
    return s["out"]


def _run_own(s):
    from paper_2605_06472_amd import binding
    if "shape" not in s:
        s["shape"] = binding.make_shape(*s["sizes"], "bf16_kv8")
    shape = s["shape"]
    if s["kind"] == "decode":
        decode = binding.paged_decode_static if s["static"] else binding.paged_decode
        decode(shape, s["q"], s["pool"], s["table"], s["prefix_lens"], s["out"])
        return s["out"]
    if s["kind"] == "prefill":
        binding.prefix_prefill(shape, s["q"], s["k_new"], s["v_new"], s["pool"], s["table"], s["prefix_lens"], s["new_lens"], s["out"])
        return s["out"]
    if s["kind"] == "write":
        binding.append_kv(shape, s["k_new"], s["v_new"], s["pool"], s["table"], s["prefix_lens"], s["new_lens"])
    binding.read_kv(shape, s["pool"], s["table"], s["prefix_lens"], s["new_lens"], s["k"], s["v"])
    return {"k": s["k"], "v": s["v"]}


# ---- the same from the definitions, in 64 bits -----------------------------------------------------------
def _e4m3_table():
    """The 256 values of e4m3: sign, four bits of exponent with bias 7, three of mantissa; no infinities, two NaN."""
    values = []
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        v = math.nan if e == 15 and m == 7 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        values.append(-v if code & 128 else v)
    return torch.tensor(values, dtype=torch.float64, device="cuda")


def exact(case, seed):
    s = prepare(case, seed)
    hkv, d, group = case["hkv"], case["d"], case["hq"] // case["hkv"]
    if case["kind"] == "write":
        def stored(x):
            # the nearest multiple of the row's step, which is 2^-3 of the value's power of two and at least 2^-9, times the row's scale
            x = x.double()
            largest = x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -126)
            power = torch.exp2(torch.ceil(torch.log2(largest / 448)).clamp(-111, 119))
            power = torch.where(largest / power > 448, power * 2, torch.where(largest / power <= 224, power / 2, power)).clamp_min(2.0 ** -111)
            y = x / power
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
            return torch.round(y / step) * step * power
        return {"k": stored(s["k_new"]), "v": stored(s["v_new"])}
    table, pool = _e4m3_table(), s["pool"]
    n_codes = 2 * hkv * PAGE * d

    def rows(kv, head, r, first, last):
        """Tokens [first, last) of request r."""
        at = torch.arange(first, last, device="cuda")
        page, slot = s["table"][r].long()[at // PAGE], at % PAGE
        byte = ((kv * hkv + head) * PAGE + slot)[:, None] * d + torch.arange(d, device="cuda")
        scale = pool[page, n_codes + (head * PAGE + slot) * 2 + kv].double()
        return table[pool[page[:, None], byte].long()] * torch.exp2(scale - 127)[:, None]

    out, at = [], 0
    for r, (p, n) in enumerate(zip(s["prefix_lens"].tolist(), s["new_lens"].tolist())):
        heads = []
        for h in range(hkv):
            if case["kind"] == "read":
                heads.append(torch.stack([rows(kv, h, r, p, p + n) for kv in range(2)]))
                continue
            k, v = rows(0, h, r, 0, p), rows(1, h, r, 0, p)
            q = (s["q"][r:r + 1] if case["kind"] == "decode" else s["q"][at:at + n])[:, h * group:(h + 1) * group].double()
            if case["kind"] == "prefill":
                k, v = torch.cat((k, s["k_new"][at:at + n, h].double())), torch.cat((v, s["v_new"][at:at + n, h].double()))
            a = torch.einsum("igd,td->igt", q, k) / math.sqrt(d)
            if case["kind"] == "prefill":
                last = p + torch.arange(n, device="cuda")
                a.masked_fill_(torch.arange(p + n, device="cuda") > last[:, None, None], -math.inf)
            heads.append(torch.einsum("igt,td->igd", torch.softmax(a, -1), v) if k.shape[0] else torch.zeros_like(q))
        out.append(torch.stack(heads, 2) if case["kind"] == "read" else torch.cat(heads, 1))
        at += n
    if case["kind"] == "read":
        both = torch.cat(out, 1)
        return {"k": both[0], "v": both[1]}
    return torch.cat(out)
