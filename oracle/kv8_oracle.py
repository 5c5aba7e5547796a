"""CPU reference of the 8-bit KV pool -- TEST INFRASTRUCTURE.

What a row of bf16 becomes (e4m3 codes and one power-of-two scale), where it stands in a page, and what the bytes of a pool stand for,
written out from the format's definition in float64.  Attention over such a pool is the fp64 oracle's over ``values(pool)``: the values
are bf16 numbers exactly.

bf16 arrays are ``uint16`` bit patterns; a pool is ``uint8`` [num_pages][page bytes].
"""
import numpy as np

P = 16
MIN_EXP, MAX_EXP, LARGEST = -111, 119, 448.0


def page_bytes(hkv, d):
    return -(-2 * hkv * P * (d + 1) // 128) * 128


def codes_of(pool, hkv, d):
    """[num_pages][2][hkv][P][d], a view."""
    return pool[:, :2 * hkv * P * d].reshape(pool.shape[0], 2, hkv, P, d)


def scales_of(pool, hkv, d):
    """[num_pages][hkv][P][2], a view (K, V)."""
    return pool[:, 2 * hkv * P * d:2 * hkv * P * (d + 1)].reshape(pool.shape[0], hkv, P, 2)


def _table():
    v = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = np.nan if (e, m) == (15, 7) else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        v[c] = -x if c & 128 else x
    return v


TABLE = _table()


def widen(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def narrow(x):
    """float64 numbers that bf16 holds -> their bits; NaN -> 0x7fc0."""
    f = np.asarray(x, np.float64).astype(np.float32)
    bits = (f.view(np.uint32) >> 16).astype(np.uint16)
    assert ((widen(bits) == x) | np.isnan(x)).all(), "not a bf16 number"
    return np.where(np.isnan(x), np.uint16(0x7fc0), bits)


def quantise(bits):
    """bf16 rows [..., d] -> codes uint8 [..., d], scale bytes uint8 [...]."""
    x = widen(bits)
    fine = np.isfinite(x)
    largest = np.where(fine, np.abs(x), 0.0).max(-1)
    e = np.full(largest.shape, MIN_EXP)
    for k in range(MIN_EXP, MAX_EXP):                   # the smallest exponent that reaches the largest value
        e = np.where(largest > LARGEST * 2.0 ** k, k + 1, e)
    y = np.where(fine, x, 0.0) * 2.0 ** -e[..., None].astype(np.float64)
    # nearest of the 127 magnitudes, ties to the even code
    mags = TABLE[:127]
    hi = np.searchsorted(mags, np.minimum(np.abs(y), LARGEST))
    lo = np.maximum(hi - 1, 0)
    below, above = np.abs(y) - mags[lo], mags[hi] - np.abs(y)
    pick = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    codes = np.where(fine, pick, 127) | np.where(np.signbit(x), 128, 0)
    return codes.astype(np.uint8), (e + 127).astype(np.uint8)


def values(pool, hkv, d):
    """What the pool's bytes stand for: bf16 bits [num_pages][2][hkv][P][d]."""
    scales = np.moveaxis(scales_of(pool, hkv, d), -1, 1).astype(np.float64) - 127     # [num_pages][2][hkv][P]
    with np.errstate(over="ignore", invalid="ignore"):
        x = TABLE[codes_of(pool, hkv, d)] * 2.0 ** scales[..., None]
    in_use = (scales >= MIN_EXP) & (scales <= MAX_EXP)
    return narrow(np.where(in_use[..., None], x, np.nan))


def append_kv(k_new, v_new, pool, block_table, prefix_lens, new_lens):
    """A copy of ``pool`` with the new rows quantised to their slots."""
    n, hkv, d = k_new.shape
    pool = np.array(pool, copy=True)
    codes, scales = codes_of(pool, hkv, d), scales_of(pool, hkv, d)
    off = 0
    for r, (p, m) in enumerate(zip(prefix_lens, new_lens)):
        pos = int(p) + np.arange(int(m))
        page, slot = np.asarray(block_table)[r, pos // P], pos % P
        for kv, src in enumerate((k_new, v_new)):
            c, s = quantise(src[off:off + int(m)])
            codes[page, kv, :, slot] = c
            scales[page, :, slot, kv] = s
        off += int(m)
    assert off == n
    return pool


def read_kv(pool, hkv, d, block_table, first_tokens, num_tokens):
    """Packed bf16 bits of the tokens [first, first + num) of every request: k, v."""
    v = values(pool, hkv, d)
    out = []
    for r, (p, m) in enumerate(zip(first_tokens, num_tokens)):
        pos = int(p) + np.arange(int(m))
        out.append(v[np.asarray(block_table)[r, pos // P], :, :, pos % P])
    both = np.concatenate(out)
    return both[:, 0], both[:, 1]
