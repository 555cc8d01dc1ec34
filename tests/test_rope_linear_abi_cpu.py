"""Refusals of the rotation, the rotating append and linear attention, without a GPU: every call fails the
host's checks, in the library and in the package, before anything is enqueued."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from paper_2604_16395_amd import _lib
from tests.test_abi_cpu import FAKE, _batch, _cache, _status

EINVAL, ERANGE, EWORKSPACE, ENOTSUP = _lib.S2L_EINVAL, _lib.S2L_ERANGE, _lib.S2L_EWORKSPACE, _lib.S2L_ENOTSUP
byref = ctypes.byref


def _rope(**kw):
    r = _lib.s2l_rope(inv_freq=FAKE, positions=None, pos_stride=0, rot_dim=128, num_axes=1, flags=0, scale=1.0)
    axes = kw.pop("axes", [])
    for k, v in kw.items():
        setattr(r, k, v)
    r.pair_axis[:len(axes)] = axes
    return r


def _qk(rope, batch, q=FAKE, qs=1024, hq=8, qo=FAKE, qos=1024, k=FAKE, ks=256, hkv=2, ko=FAKE, kos=256):
    return _status("s2l_rope_qk", byref(batch) if batch else None, byref(rope) if rope else None, q, qs, hq, qo, qos, k, ks, hkv,
                   ko, kos, None)


def _append(rope, batch, cache, q=FAKE, qs=1024, hq=8, qo=FAKE, qos=1024, k=FAKE, ks=256, v=FAKE, vs=256):
    return _status("s2l_rope_kv_append", byref(cache) if cache else None, byref(batch) if batch else None,
                   byref(rope) if rope else None, q, qs, hq, qo, qos, k, ks, v, vs, None)


BAD_ROPES = [
    (dict(inv_freq=None), EINVAL), (dict(rot_dim=0), ENOTSUP), (dict(rot_dim=24), ENOTSUP), (dict(rot_dim=144), ENOTSUP),
    (dict(num_axes=0), ENOTSUP), (dict(num_axes=5, positions=FAKE, pos_stride=99), ENOTSUP), (dict(flags=2), EINVAL),
    (dict(scale=0.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(num_axes=2), EINVAL),
    (dict(num_axes=2, positions=FAKE, pos_stride=3), EINVAL), (dict(axes=[0, 1]), EINVAL),
    (dict(num_axes=2, positions=FAKE, pos_stride=4, axes=[0, 2]), EINVAL),
]


@pytest.mark.parametrize("kw,status", BAD_ROPES)
def test_bad_rotations(kw, status):
    b, keep = _batch([3], [4])
    st, msg = _qk(_rope(**kw), b)
    assert st == status and msg
    st, msg = _append(_rope(**kw), b, _cache())
    assert st == status and msg


@pytest.mark.parametrize("kw", [dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(qs=-1), dict(ks=1 << 40),
                                dict(qos=1023), dict(kos=255), dict(hq=-1), dict(hkv=-1), dict(q=FAKE + 1), dict(ko=FAKE + 1),
                                dict(qs=2048)])    # q in place needs one stride
def test_bad_rows(kw):
    b, keep = _batch([3], [4])
    st, msg = _qk(_rope(), b, **kw)
    assert st == EINVAL and msg


def test_null_structs_and_lengths():
    b, keep = _batch([3], [4])
    assert _qk(None, b)[0] == EINVAL and _qk(_rope(), None)[0] == EINVAL
    assert _append(_rope(), b, None)[0] == EINVAL and _append(None, b, _cache())[0] == EINVAL
    assert _append(_rope(), b, _cache(), v=None)[0] == EINVAL and _append(_rope(), b, _cache(), vs=-2)[0] == EINVAL
    assert _append(_rope(), b, _cache(head_dim=64))[0] == ENOTSUP and _append(_rope(), b, _cache(dtype=1))[0] == EINVAL
    assert _qk(_rope(), b, hq=65536, qs=1 << 24, qos=1 << 24)[0] == ENOTSUP
    for P, C, status in (([-1], [4], EINVAL), ([0], [-1], EINVAL), ([1 << 30], [1], EINVAL)):
        bad, keep2 = _batch(P, C)
        assert _qk(_rope(), bad)[0] == status
    bad, keep2 = _batch([1000], [25])
    assert _append(_rope(), bad, _cache())[0] == ERANGE
    b.cu_chunk = None
    assert _qk(_rope(), b)[0] == EINVAL and _append(_rope(), b, _cache())[0] == EINVAL


def test_rows_beyond_one_launch():
    b, keep = _batch([0, 0], [1 << 25, 1 << 25])
    assert _qk(_rope(), b, hq=14, hkv=2, qs=2048, qos=2048)[0] == ENOTSUP
    b, keep = _batch([0] * 8, [1 << 23] * 8, max_pages=1 << 20)
    assert _append(_rope(), b, _cache())[0] == ENOTSUP


def _linear(state, batch, q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, hkv=2, scale=0.1, out=FAKE, os_=1024, ws=FAKE, n=1 << 40):
    return _status("s2l_linear_attn", byref(state) if state else None, byref(batch) if batch else None, q, qs, k, ks, v, vs, hkv,
                   scale, out, os_, ws, n, None)


def _state(**kw):
    s = _lib.s2l_linear_state(states=FAKE, log_decay=FAKE, slot_in=FAKE, slot_out=FAKE, num_slots=4, num_heads=8)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("kw,status", [
    (dict(states=None), EINVAL), (dict(log_decay=None), EINVAL), (dict(slot_in=None), EINVAL), (dict(slot_out=None), EINVAL),
    (dict(num_slots=0), EINVAL), (dict(num_heads=0), EINVAL), (dict(num_heads=7), EINVAL), (dict(num_heads=65538), ENOTSUP),
    (dict(states=FAKE + 4), EINVAL),
])
def test_bad_states(kw, status):
    b, keep = _batch([3], [4])
    st, msg = _linear(_state(**kw), b)
    assert st == status and msg


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(qs=-1), dict(vs=-1), dict(os_=1023),
                                dict(hkv=0), dict(hkv=3), dict(scale=float("inf")), dict(out=FAKE + 1)])
def test_bad_linear_arguments(kw):
    b, keep = _batch([3], [4])
    st, msg = _linear(_state(), b, **kw)
    assert st == EINVAL and msg


def test_linear_null_structs_and_sizes():
    b, keep = _batch([3], [4])
    assert _linear(None, b)[0] == EINVAL and _linear(_state(), None)[0] == EINVAL
    n = ctypes.c_size_t()
    assert _status("s2l_linear_attn_workspace_bytes", byref(b), 8, None)[0] == EINVAL
    assert _status("s2l_linear_attn_workspace_bytes", byref(b), 0, byref(n))[0] == EINVAL
    assert _status("s2l_linear_attn_workspace_bytes", None, 8, byref(n))[0] == EINVAL
    b.chunk_lens = None
    assert _linear(_state(), b)[0] == EINVAL


def test_linear_heads_beyond_one_launch_and_outputs_in_place():
    b, keep = _batch([0] * 1025, [1] * 1025)
    st, msg = _linear(_state(num_heads=8192), b, qs=1 << 20, os_=1 << 20)
    assert st == ENOTSUP and msg
    b, keep = _batch([0], [4])
    other = FAKE + 4096
    for kw in (dict(k=other, v=other), dict(q=other, v=other), dict(q=other, k=other)):
        st, msg = _linear(_state(), b, **kw)
        assert st == EINVAL and "out must not be" in msg


def test_pair_axes():
    assert s2l.rope_pair_axes((2, 1, 1)) == [0, 0, 1, 2]
    assert s2l.rope_pair_axes((4, 2, 2), cyclic=True) == [0, 1, 2, 0, 1, 2, 0, 0]
    for bad in ((), (-1, 2)):
        with pytest.raises(ValueError):
            s2l.rope_pair_axes(bad)
    with pytest.raises(ValueError):
        s2l.rope_pair_axes((0, 4), cyclic=True)


def test_the_package_refuses_what_it_cannot_pass_on():
    """Types, shapes, strides, missing rows, and tensors that are not on the batch's GPU."""
    batch = s2l.Batch([16], [4], np.zeros((1, 2), np.int32), device="cpu")
    inv, q, k = torch.ones(64), torch.zeros((4, 8, 128), dtype=torch.bfloat16), torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    for bad in (q.float(), q[..., :64], q.transpose(0, 1), q[:3], q.repeat_interleave(2, 2)[..., ::2], q):   # the last: a CPU tensor
        with pytest.raises(ValueError, match="q "):
            s2l.s2l_rope_qk(batch, s2l.Rope(inv), bad, q, stream=0)
    for kw in (dict(pair_axes=[0] * 63), dict(pair_axes=[4] * 64), dict(pair_axes=[-1] * 64)):
        with pytest.raises(ValueError):
            s2l.Rope(inv, **kw)
    for bad in (torch.ones(65), torch.ones((2, 8)), torch.ones(64, dtype=torch.float64)):
        with pytest.raises(ValueError):
            s2l.Rope(bad)
    for bad in (torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int64), torch.zeros((4, 2), dtype=torch.int32).t()):
        with pytest.raises(ValueError):
            s2l.Rope(inv, bad).c(4, inv.device)
    states, decay, slots = torch.zeros((2, 8, 128, 128)), torch.zeros(8), torch.zeros(1, dtype=torch.int32)
    for bad in ((states.half(), decay), (states, decay[:7]), (states[..., :64].contiguous(), decay)):
        with pytest.raises(ValueError):
            s2l.LinearState(*bad, slots, slots)
    for bad in (slots.long(), torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError):
            s2l.LinearState(states, decay, bad, slots).c(1, states.device)
    # attributes exchanged after the checks of the constructor
    state, rope = s2l.LinearState(states, decay, slots, slots), s2l.Rope(inv)
    state.states, rope.inv_freq = states[:, :4], inv.double()
    for obj, n in ((state, 1), (rope, 4)):
        with pytest.raises(ValueError):
            obj.c(n, inv.device)
    with pytest.raises(ValueError):
        s2l.s2l_linear_attn(s2l.LinearState(states, decay, slots, slots), batch, q, k, k, 0.1, q, None, 0)
    with pytest.raises(ValueError):
        s2l.s2l_rope_kv_append(None, batch, s2l.Rope(inv), None, None, k, k, 0)
