"""Calls of the rotation, the rotating append and linear attention without a GPU: what is asked of arguments that a call
does not read, and of those on other devices."""
import contextlib
import types

import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from paper_2604_16395_amd import _lib
from tests.test_abi_cpu import _batch
from tests.test_rope_linear_abi_cpu import _linear, _qk, _rope, _state


@pytest.mark.parametrize("name", ["prefix_lens", "block_tables"])
def test_linear_attention_asks_for_no_array_that_it_does_not_read(name):
    """The batch is taken: what is refused next is the scale."""
    b, keep = _batch([3], [4])
    setattr(b, name, None)
    st, msg = _linear(_state(), b, scale=float("inf"))
    assert st == _lib.S2L_EINVAL and msg == "scale must be finite"


@pytest.mark.parametrize("name", ["chunk_lens", "cu_chunk", "prefix_lens_host", "chunk_lens_host"])
def test_linear_attention_asks_for_the_arrays_that_it_reads(name):
    b, keep = _batch([3], [4])
    setattr(b, name, None)
    st, msg = _linear(_state(), b)
    assert st == _lib.S2L_EINVAL and "NULL" in msg


def test_the_rotation_asks_for_prefix_lengths():
    b, keep = _batch([3], [4])
    b.prefix_lens = None
    st, msg = _qk(_rope(), b)
    assert st == _lib.S2L_EINVAL and "NULL" in msg


@pytest.mark.parametrize("device,current", [("cuda:1", ["cuda:1"]), ("cuda:0", ["cuda:0"]), ("cpu", [])])
def test_workspaces_are_sized_on_the_batch_s_device(monkeypatch, device, current):
    """As the call itself runs there: another device current may have another number of CUs."""
    seen, now = [], []

    @contextlib.contextmanager
    def use(d):
        now.append(str(d))
        yield
        now.pop()

    b, keep = _batch([3], [4])
    batch = types.SimpleNamespace(c=lambda: b, chunk_lens=types.SimpleNamespace(device=torch.device(device)))
    monkeypatch.setattr(torch.cuda, "device", use)
    monkeypatch.setattr(_lib, "call", lambda name, *args: seen.append((name, list(now))))
    assert s2l.s2l_linear_attn_workspace_bytes(batch, 8) == 0
    assert seen == [("s2l_linear_attn_workspace_bytes", current)]


@pytest.mark.parametrize("away", ["k_pages", "v_pages", "k_scale", "v_scale"])
def test_the_rotating_append_refuses_a_cache_on_another_device(monkeypatch, away):
    """Its kernel would write through a pointer that is not of its device."""
    batch = s2l.Batch([16], [4], np.zeros((1, 2), np.int32), device="cpu")
    pages = [torch.zeros((2, 2, 16, 128), dtype=torch.uint8, device="meta" if away == n else "cpu") for n in ("k_pages", "v_pages")]
    scales = [torch.ones(2, device="meta" if away == n else "cpu") for n in ("k_scale", "v_scale")]
    rows = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    monkeypatch.setattr(s2l, "_rows", lambda t, name, batch: (None, 256, t.shape[1]))   # as of tensors on the batch's GPU
    monkeypatch.setattr(s2l, "_call_on", lambda *args, **kw: None)
    with pytest.raises(ValueError, match=f"{away} is on meta"):
        s2l.s2l_rope_kv_append(s2l.PagedKVCache(*pages, *scales), batch, s2l.Rope(torch.ones(64)), None, None, rows, rows, 0)
    fine = s2l.PagedKVCache(*(torch.zeros((2, 2, 16, 128), dtype=torch.bfloat16) for _ in range(2)))
    s2l.s2l_rope_kv_append(fine, batch, s2l.Rope(torch.ones(64)), None, None, rows, rows, 0)
