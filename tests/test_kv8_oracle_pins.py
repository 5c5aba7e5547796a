"""The CPU reference of the 8-bit pool against what it has to agree with: torch's e4m3 type, the format's error bounds, the layout in the
header's words, and its own inverse."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as K8
from paper_2605_06472_amd import binding, workloads as W


def _rows(seed, n, d, spread):
    rng = np.random.default_rng(seed)
    return W.f32_to_bf16_bits((rng.standard_normal((n, d)) * 2.0 ** rng.integers(-spread, spread + 1, (n, 1))).astype(np.float32))


def test_the_table_is_e4m3():
    want = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(K8.TABLE, want, equal_nan=True)


@pytest.mark.parametrize("d", [64, 128])
def test_codes_are_the_nearest(d):
    bits = _rows(5, 400, d, 100)
    bits[0] = 0
    bits[1] = 0x8000                                        # minus zero
    bits[2, ::2] = np.arange(d // 2) + 1                    # subnormal bf16
    codes, scale = K8.quantise(bits)
    x, e = K8.widen(bits), scale.astype(int) - 127
    # torch rounds to the nearest e4m3 number, ties to even
    y = torch.from_numpy(x * 2.0 ** -e[:, None].astype(np.float64)).float()
    assert np.array_equal(codes, y.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    # the smallest scale that holds the row, and the bound that the header states
    top = np.abs(x).max(-1)
    assert (top <= 448 * 2.0 ** e).all() and ((top > 448 * 2.0 ** (e - 1)) | (e == K8.MIN_EXP)).all()
    off = np.abs(K8.TABLE[codes] * 2.0 ** e[:, None].astype(np.float64) - x)
    assert (off <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** (e[:, None] - 10.0))).all()


def test_infinities_nan_and_the_largest_numbers():
    bits = _rows(6, 4, 64, 0)
    bits[0, 3], bits[0, 9] = 0x7f80, 0xff80                 # infinities
    bits[1, 7] = 0xffc1                                     # NaN
    bits[2, :] = 0x7f7f                                     # the largest bf16 number: saturates
    bits[3, :] = 0xff80                                     # nothing finite
    codes, scale = K8.quantise(bits)
    v = K8.TABLE[codes]
    assert np.isnan(v[0, [3, 9]]).all() and np.isfinite(np.delete(v[0], [3, 9])).all() and np.isnan(v[1, 7])
    assert (v[2] == 448).all() and scale[2] == 246 and np.isnan(v[3]).all() and scale[3] == 16
    assert (scale[:2] < 140).all()                          # what is not finite does not set the scale


@pytest.mark.parametrize("hkv,d", [(1, 64), (2, 64), (1, 128), (3, 128), (8, 128)])
def test_layout_and_the_way_back(hkv, d):
    nbytes = K8.page_bytes(hkv, d)
    assert nbytes % 128 == 0 and 0 <= nbytes - 2 * hkv * 16 * (d + 1) < 128
    assert nbytes == binding.page_bytes(binding.make_shape(1, hkv, hkv, d, 16, 4, 1, "bf16_kv8"))
    b = W.ragged_small(31, "bf16", Hq=hkv, Hkv=hkv, d=d)
    before = np.full((b.num_pages, nbytes), 0xA5, np.uint8)
    pool = K8.append_kv(b.k_new, b.v_new, before, b.block_table, b.prefix_lens, b.new_lens)
    # one token by hand: byte addresses from the header
    r, t, kv, g = 2, 17, 1, hkv - 1
    pos = int(b.prefix_lens[r]) + t
    page, slot = pool[b.block_table[r, pos // 16]], pos % 16
    row = b.v_new[int(b.new_lens[:r].sum()) + t, g]
    codes, scale = K8.quantise(row)
    at = ((kv * hkv + g) * 16 + slot) * d
    assert np.array_equal(page[at:at + d], codes) and page[2 * hkv * 16 * d + (g * 16 + slot) * 2 + kv] == scale
    assert (pool[:, 2 * hkv * 16 * (d + 1):] == 0xA5).all()
    changed = int((pool != before).any(1).sum())
    assert changed <= sum(-(-(int(p) + int(n)) // 16) for p, n in zip(b.prefix_lens, b.new_lens))
    # read back, appended again: the same values
    k, v = K8.read_kv(pool, hkv, d, b.block_table, b.prefix_lens, b.new_lens)
    again = K8.append_kv(k, v, before, b.block_table, b.prefix_lens, b.new_lens)
    k2, v2 = K8.read_kv(again, hkv, d, b.block_table, b.prefix_lens, b.new_lens)
    assert np.array_equal(k, k2) and np.array_equal(v, v2)


MISTAKES = {
    "scale one too small": lambda c, s: (c, s - 1),
    "codes of the neighbour": lambda c, s: (np.roll(c, 1, -1), s),
    "truncated": lambda c, s: (np.where(c & 1, c - 1, c), s),
    "sign lost": lambda c, s: (c & 127, s),
}


@pytest.mark.parametrize("name", sorted(MISTAKES))
def test_planted_mistakes_are_seen(name, monkeypatch):
    plain = K8.quantise
    monkeypatch.setattr(K8, "quantise", lambda bits: MISTAKES[name](*plain(bits)))
    with pytest.raises(AssertionError):
        test_codes_are_the_nearest(64)
