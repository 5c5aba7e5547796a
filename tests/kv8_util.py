"""A bf16 batch whose pool is held in 8 bits: the same logical rows quantised by the CPU reference, every slot that holds no prefix token
filled with bytes that must not be looked at (NaN codes under a scale that no append writes)."""
import dataclasses

import numpy as np
import torch

from oracle import kv8_oracle as K8
from paper_2605_06472_amd import binding, workloads as W
from tests.gpu_util import to_numpy, to_torch


@dataclasses.dataclass
class Kv8Batch:
    b: W.Batch
    pool: np.ndarray          # uint8 [num_pages][page bytes]

    @property
    def values(self):
        """bf16 bits of a bf16 pool that holds the same values."""
        return K8.values(self.pool, self.b.Hkv, self.b.d)


def held_slots(b):
    live = np.zeros((b.num_pages, b.P), bool)
    for r in range(b.B):
        pos = np.arange(int(b.prefix_lens[r]))
        live[b.block_table[r, pos // b.P], pos % b.P] = True
    return live


def make(b: W.Batch) -> Kv8Batch:
    pool = np.full((b.num_pages, K8.page_bytes(b.Hkv, b.d)), 0xFF, np.uint8)
    codes, scales = K8.quantise(b.kv_pool)
    live = held_slots(b)
    K8.codes_of(pool, b.Hkv, b.d)[:] = np.where(live[:, None, None, :, None], codes, 0xFF)
    K8.scales_of(pool, b.Hkv, b.d)[:] = np.where(live[:, None, :, None], np.moveaxis(scales, 1, -1), 0xFF)
    return Kv8Batch(b, pool)


class DeviceKv8:
    """On the GPU, with the calls of the binding."""

    def __init__(self, kb: Kv8Batch):
        b = self.b = kb.b
        self.shape = self.shape_of("bf16_kv8")
        self.q, self.k_new, self.v_new, self.block_table = (to_torch(a) for a in (b.q, b.k_new, b.v_new, b.block_table))
        self.pool = torch.from_numpy(kb.pool.copy()).cuda()
        self.plain = to_torch(np.ascontiguousarray(kb.values))          # the bf16 pool of the same values
        self.out = torch.zeros_like(self.q)

    def shape_of(self, dtype, batch=None):
        b = self.b
        return binding.make_shape(b.B if batch is None else batch, b.Hq, b.Hkv, b.d, b.P, b.num_pages, b.max_pages, dtype)

    def prefill(self, plain=False, stream=None):
        b, out = self.b, torch.full_like(self.q, 7.0)
        binding.prefix_prefill(self.shape_of("bf16") if plain else self.shape, self.q, self.k_new, self.v_new, self.plain if plain else self.pool,
                               self.block_table, b.prefix_lens, b.new_lens, out, stream)
        return out

    def decode(self, lens=None, static=False, stream=None):
        out = torch.full_like(self.q, 7.0)
        call = binding.paged_decode_static if static else binding.paged_decode
        call(self.shape, self.q, self.pool, self.block_table, self.b.prefix_lens if lens is None else np.asarray(lens, np.int32), out, stream)
        return out

    def append(self, stream=None):
        b = self.b
        binding.append_kv(self.shape, self.k_new, self.v_new, self.pool, self.block_table, b.prefix_lens, b.new_lens, stream)


def f64(t):
    torch.cuda.synchronize()
    return W.to_f64(to_numpy(t))
