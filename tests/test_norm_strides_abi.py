"""Strides that the norm's backward is given for the gradients it writes, without a GPU: what is refused."""

import ctypes

import pytest
import torch

from paper_2508_10774_amd import binding

FAKE = ctypes.c_void_p(0x10000)      # (never dereferenced: the calls are refused first)
INVALID, WORKSPACE = -1, -3


def _params(**kw):
    base = dict(B=2, H=4, L=100, d=64, block=64)
    base.update(kw)
    return ctypes.byref(binding.Params(**base).c())


def _norm(**kw):
    n = binding.asa_qk_norm(H_kv=2, eps=1e-6)
    for k, v in kw.items():
        setattr(n, k, (ctypes.c_int64 * 3)(*v))
    return ctypes.byref(n)


def _bwd(p, n):
    """No workspace: a call whose strides are in order ends with that."""
    return binding.load().asa_qk_norm_rope_bwd(p, n, *[FAKE] * 8, None, None, None, 0, None)


def test_strides_of_the_gradients():
    apart = (25600, 64, 256)                                          # [B, L, heads, d]
    assert _bwd(_params(), _norm(dq_stride=apart, dk_stride=(12800, 64, 128))) == WORKSPACE
    assert _bwd(_params(q_stride=apart), _norm(dq_stride=(25600, 6400, 64))) == WORKSPACE
    for which in ("dq_stride", "dk_stride"):
        for bad in ((25600, 4, 256), (25600, 64, 60), (-25600, 64, 256), (0, 64, 256), (25600, 0, 256), (25600, 64, 120),
                    (25600, 6392, 64), (25600, 64, 1 << 24)):
            assert _bwd(_params(), _norm(**{which: bad})) == INVALID, (which, bad)


def test_rows_of_q_and_k_may_repeat_where_the_gradients_lie_apart():
    p = _params(q_stride=(0, 6400, 64), k_stride=(6400, 0, 64))
    assert _bwd(p, _norm()) == INVALID                                # (gradients laid out as q and k)
    assert _bwd(p, _norm(dq_stride=(25600, 6400, 64), dk_stride=(12800, 6400, 64))) == WORKSPACE
    ws = binding.load().asa_qk_norm_rope_bwd_workspace_bytes
    assert ws(p, _norm()) == ws(_params(), _norm()) > 0               # (sizes alone decide)


def test_the_bindings_strides_of_a_gradient():
    shape = (2, 3, 5, 64)
    t = torch.zeros(2, 5, 4, 64, dtype=torch.bfloat16)[:, :, :3].transpose(1, 2)
    assert binding._own_strides(t, "dq", shape) == (5 * 4 * 64, 64, 4 * 64)
    one = torch.zeros(1, 64, dtype=torch.bfloat16).as_strided((1, 1, 1, 64), (7, 3, 1, 1))
    strides = binding._own_strides(one, "dq", (1, 1, 1, 64))      # (a stride over one element says nothing)
    assert all(s % 8 == 0 and s >= 64 for s in strides)
    for bad in (torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16).expand(shape), torch.zeros(2, 3, 5, 128, dtype=torch.bfloat16)[..., ::2],
                torch.zeros(2, 1, 5, 64, dtype=torch.bfloat16).expand(shape)):
        with pytest.raises(binding.AsaError, match="dq: strides"):
            binding._own_strides(bad, "dq", shape)
    assert binding._own_strides(None, "dk", shape) == (0, 0, 0)
