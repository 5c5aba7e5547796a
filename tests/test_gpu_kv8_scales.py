"""Attention over 8-bit pools whose rows have scales at and near both ends, 2^-111 and 2^119: keys against queries that make ordinary scores of them,
values as they are."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import kv8_oracle as K8                                              # noqa: E402
from paper_2605_06472_amd import binding, workloads as W                         # noqa: E402
from tests.kv8_util import DeviceKv8, f64, make                                  # noqa: E402
from tests.test_gpu_kv8 import prefill_close                                     # noqa: E402

HEADS = [(8, 2, 128), (16, 2, 64), (32, 2, 128), (4, 4, 64)]


def _times(bits, e):
    with np.errstate(over="raise"):
        return W.f32_to_bf16_bits((W.to_f64(bits) * 2.0 ** e).astype(np.float32))


def _batch(seed, heads, k=0, v=0, **kw):
    """Keys times 2^k, queries times 2^-k, values times 2^v."""
    hq, hkv, d = heads
    kw = kw or dict(prefix_lens=(700, 33, 4097, 1), new_lens=(1, 40, 3, 20), num_pages=400)
    b = W.ragged_small(seed, "bf16", Hq=hq, Hkv=hkv, d=d, **kw)
    b.q = _times(b.q, -k)
    b.k_new, b.v_new = _times(b.k_new, k), _times(b.v_new, v)
    b.kv_pool = np.stack([_times(b.kv_pool[:, 0], k), _times(b.kv_pool[:, 1], v)], 1)
    return b


def _scales(kb, kv):
    s = K8.scales_of(kb.pool, kb.b.Hkv, kb.b.d)[..., kv].astype(int)
    return s[s != 0xFF] - 127


def _both_attentions(oracle, kb):
    """Decode: half a step of bf16 (2^-8 of the result); scores, weights and sums in fp32, as a sum over the context of what each term may be off by:
    its score (d + 8 roundings of at most the largest score, twice 2^-24 of it with the exponential's), its weight's two bf16 halves (2^-17 of it, or where the
    product of weight and scale is below what bf16 holds in full, 2^-134, times codes of at most 448), its sum."""
    b, d = kb.b, DeviceKv8(kb)
    lens = b.prefix_lens
    want = oracle.decode(b.q[:b.B], kb.values, b.block_table, lens)
    d.q = d.q[:b.B].contiguous()
    got = d.decode()
    assert torch.equal(got, d.decode(static=True))
    vals = np.abs(np.nan_to_num(W.to_f64(kb.values)))
    top = np.sqrt((W.to_f64(b.q[:b.B]) ** 2).sum(-1).max() * (vals[:, 0] ** 2).sum(-1).max() / b.d)
    vmax = vals[:, 1].max()
    off = vmax * (2 * 2.0 ** -24 * ((b.d + 8) * top + max(lens)) + 2.0 ** -16) + max(lens) * 2.0 ** -134 * 448
    out = f64(got)
    assert np.isfinite(out).all()
    err = np.abs(out - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + off).all(), "decode: %.3e of %.3e" % ((err - 2.0 ** -8 * np.abs(want)).max(), off)
    d = DeviceKv8(kb)
    want = oracle.prefill(b.q, b.k_new, b.v_new, kb.values, b.block_table, b.prefix_lens, b.new_lens)
    try:
        for waves in (0, 4, 64):
            binding.set_attn_waves(waves)
            prefill_close(f64(d.prefill()) / vmax, want / vmax, "prefill, %d waves" % waves)
    finally:
        binding.set_attn_waves(0)


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("v", [-112, -104, -100, 105])
def test_values(oracle, heads, v):
    kb = make(_batch(340, heads, v=v))
    assert _scales(kb, 1).min() == -111 if v <= -104 else _scales(kb, 1).max() in (v - 8, v - 7, v - 6)
    _both_attentions(oracle, kb)


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("k", [-108, -104, 118, 124])
def test_keys(oracle, heads, k):
    kb = make(_batch(341, heads, k=k))
    assert _scales(kb, 0).min() == -111 if k < 0 else _scales(kb, 0).max() >= k - 7
    _both_attentions(oracle, kb)


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
def test_the_largest_numbers_come_through_alone(heads):
    """A context of one token is that token's value, up to the largest code of the largest scale."""
    b = _batch(342, heads, prefix_lens=(1, 1, 1), new_lens=(1, 1, 1), num_pages=40)
    page = b.block_table[:, 0]
    rng = np.random.default_rng(7)
    b.kv_pool[page, 1, :, 0] = rng.choice([0x7f7f, 0x7f60, 0x7f00, 0x7e80, 0xff7f, 0xff60, 0xfe12], b.kv_pool[page, 1, :, 0].shape).astype(np.uint16)
    kb = make(b)
    assert _scales(kb, 1).max() == 119
    got = f64(DeviceKv8(kb).decode())
    want = np.repeat(W.to_f64(kb.values)[page, 1, :, 0], b.Hq // b.Hkv, 1)
    assert np.isfinite(want).all() and np.array_equal(got, want)
