"""A model's own norm weights are nn.Parameters: the native marshalling takes them as it takes plain tensors (CPU: torch
says that its current device is -1, where CPU tensors are, and the library refuses the eps of 0)."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from paper_2604_16395_amd import _lib


@pytest.fixture
def native(monkeypatch):
    try:
        monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
        s2l._native = None
        yield s2l._load_native()
    finally:   # the module holds what it was set up with
        monkeypatch.undo()
        s2l._native = None
        s2l._load_native()


class Other(torch.Tensor):
    pass


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("stream", [0, None])
def test_parameters_are_marshalled_natively(native, dtype, stream):
    batch, rope = s2l.Batch([16], [4], np.zeros((1, 2), np.int32), device="cpu"), s2l.Rope(torch.ones(64))
    row = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    cache = s2l.PagedKVCache(*(torch.zeros((2, 2, s2l.MXFP4_RUN_BYTES), dtype=torch.uint8) for _ in "kv"))
    plain, model = torch.ones(128, dtype=dtype), torch.nn.RMSNorm(128, dtype=dtype).weight
    assert type(model) is torch.nn.Parameter

    def taken(norm):
        one = native.norm_rope_qk(batch, norm, rope, row, row, row, row, stream)
        assert one == native.norm_rope_append(cache, batch, norm, rope, row, row, row, row, stream)
        return one

    for q, k in ((plain, plain), (model, model), (model, None), (None, model), (plain, model), (torch.nn.Parameter(plain, False), model)):
        norm = s2l.QKNorm(q, k, 0.0)
        assert taken(norm) == _lib.S2L_EINVAL
        with pytest.raises(s2l.S2LError, match="eps"):
            s2l.s2l_norm_rope_qk(batch, norm, rope, row, row, row, row, stream)
    other = torch.bfloat16 if dtype == torch.float32 else torch.float32
    for wrong in (torch.nn.Parameter(torch.ones(256, dtype=dtype)[::2]), torch.nn.Parameter(torch.ones(64, dtype=dtype)),
                  torch.nn.Parameter(torch.ones(1, 128, dtype=dtype)), torch.nn.Parameter(torch.ones(128, dtype=other)), plain.as_subclass(Other)):
        norm = s2l.QKNorm(plain, plain, 0.0)
        norm.k_weight = wrong
        assert taken(norm) is None       # the general path says what is wrong, or takes it
