"""Helpers of the GPU tests of MXFP4 caches: cases whose keys and values are MXFP4 values (which bf16 holds
exactly, so that the oracle of bf16 pages answers for them), and their pools."""
import numpy as np
import torch

import paper_2604_16395_amd as s2l
import workloads
from oracle import mxfp4
from oracle.paged_kv import bf16_bits_to_f32, ref_append
from tests.gpu_util import DEV, Setup, to_bf16


def to_f64(bits):
    """bf16 bits -> float64, NaNs among them."""
    with np.errstate(invalid="ignore"):
        return bf16_bits_to_f32(bits).astype(np.float64)


def quantised_bits(bits):
    """bf16 bits [...][128] -> the bf16 bits of their MXFP4 values."""
    return workloads.bf16_bits(mxfp4.dequantise(*mxfp4.quantise(bf16_bits_to_f32(bits))).astype(np.float32))


def mx_case(*args, **kw):
    case = workloads.make_case(*args, **kw)
    case.k_full_bits, case.v_full_bits = quantised_bits(case.k_full_bits), quantised_bits(case.v_full_bits)
    return case


class MxSetup(Setup):
    """Setup with MXFP4 pools: the prefix encoded by the oracle (poison and unwritten slots NaN), the
    chunk appended by the GPU.  The raw chunk rows are the case's, already on the grid."""

    def __init__(self, case, block_tables=None):
        super().__init__(case, block_tables)
        self.cache = s2l.PagedKVCache(*(torch.from_numpy(mxfp4.from_rows(to_f64(p))).to(DEV) for p in (self.kp_ref, self.vp_ref)))

    def append(self):
        s2l.s2l_kv_append(self.cache, self.batch, to_bf16(self.k_new), to_bf16(self.v_new))
        ref_append(self.kp_ref, self.vp_ref, self.tables, self.case.prefix_lens, self.case.chunk_lens,
                   self.case.cu_chunk, self.k_new, self.v_new)
        self.appended = True


def slots(tables, r, positions):
    """(pages, slots) of positions of request r."""
    p = np.asarray(positions, dtype=np.int64)
    return [int(x) for x in np.asarray(tables[r])[p // 16]], [int(x) for x in p % 16]
