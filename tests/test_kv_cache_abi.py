"""What the norm, cache and cached-attention calls refuse, without a GPU, and pins of their oracle."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import kv_cache as ref
from paper_2508_10774_amd import binding

FAKE = ctypes.c_void_p(0x10000)      # (never dereferenced: the calls are refused first)
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


def _params(**kw):
    base = dict(B=2, H=4, L=100, d=64, block=64)
    base.update(kw)
    return ctypes.byref(binding.Params(**base).c())


def _norm(**kw):
    n = binding.asa_qk_norm(H_kv=2, kind=0, eps=1e-6, rot_dim=32, pairing=0, table_rows=10, cos_table=0x1000, sin_table=0x2000)
    for k, v in kw.items():
        setattr(n, k, (ctypes.c_int64 * 3)(*v) if isinstance(v, tuple) else v)
    return ctypes.byref(n)


def _cache(**kw):
    c = binding.asa_kv_cache(H_kv=2, max_blocks=8, k=0x1000, v=0x2000, k_scale=0x3000, v_scale=0x4000)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def test_norm_refusals():
    L = binding.load()
    fwd = lambda p, n, q=FAKE, k=FAKE, qo=FAKE, ko=FAKE: L.asa_qk_norm_rope(p, n, q, k, qo, ko, None)
    ws = L.asa_qk_norm_rope_bwd_workspace_bytes
    assert ws(_params(), _norm()) > 0 and ws(_params(), _norm()) % 256 == 0
    for bad in (dict(kind=2), dict(kind=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(rot_dim=8),
                dict(rot_dim=80), dict(rot_dim=-16), dict(pairing=2), dict(table_rows=0), dict(cos_table=None), dict(sin_table=0x2004),
                dict(H_kv=-1), dict(q_bias=0x100), dict(k_bias=0x100), dict(start=0x101), dict(q_weight=0x102),
                dict(q_out_stride=(0, 0, 60)), dict(k_out_stride=(8, 4, 64))):
        assert fwd(_params(), _norm(**bad)) == INVALID, bad
        assert ws(_params(), _norm(**bad)) == 0, bad
    for bad in (dict(L=0), dict(B=0), dict(H=0), dict(q_stride=(1, 8, 64)), dict(k_stride=(0, 0, 32))):
        assert fwd(_params(**bad), _norm()) == INVALID, bad
    for bad in (dict(d=96), dict(L=131073), dict(B=1 << 30)):
        assert fwd(_params(**bad), _norm()) == UNSUPPORTED, bad
    odd = ctypes.c_void_p(0x10008)
    assert fwd(None, _norm()) == fwd(_params(), None) == INVALID
    for args in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(q=odd), dict(k=odd), dict(qo=odd), dict(ko=odd)):
        assert fwd(_params(), _norm(), **args) == INVALID, args

    def bwd(n=_norm(), q=FAKE, k=FAKE, gq=FAKE, gk=FAKE, dq=FAKE, dk=FAKE, qw=FAKE, kw=FAKE, qb=None, kb=None, w=FAKE, size=1 << 30):
        return L.asa_qk_norm_rope_bwd(_params(), n, q, k, gq, gk, dq, dk, qw, kw, qb, kb, w, size, None)

    for args in (dict(q=None), dict(k=None), dict(gq=None), dict(gk=None), dict(dq=None), dict(dk=None), dict(qb=FAKE), dict(kb=FAKE),
                 dict(k=None, gk=None, dk=None), dict(qw=ctypes.c_void_p(0x10002)), dict(gq=odd), dict(dk=odd)):
        assert bwd(**args) == INVALID, args
    # rows that are written lie apart: a stride of 0, heads inside one another, tokens inside a head
    for bad in ((0, 6400, 64), ((1 << 62) + 8, 1 << 62, 64), (25600, 0, 64), (25600, 64, 64), (25600, 6392, 64)):
        assert fwd(_params(), _norm(q_out_stride=bad)) == INVALID, bad
        assert L.asa_qk_norm_rope_bwd(_params(q_stride=bad), _norm(), *[FAKE] * 8, None, None, None, 0, None) == INVALID, bad
    need = ws(_params(), _norm())
    assert bwd(w=None) == bwd(size=need - 1) == bwd(w=odd) == WORKSPACE


def test_cache_refusals():
    L = binding.load()
    for fn in (L.asa_cache_write, L.asa_cache_read):
        call = lambda p=_params(), c=_cache(), k=FAKE, v=FAKE, s=None, n=None: fn(p, c, k, v, s, n, None)
        assert call(p=None) == call(c=None) == call(k=None, v=None) == INVALID
        for bad in (dict(H_kv=0), dict(max_blocks=0), dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=0x4002), dict(v=0x2008)):
            assert call(c=_cache(**bad)) == INVALID, bad
        assert call(c=_cache(max_blocks=65537)) == UNSUPPORTED
        for bad in (dict(L=0), dict(B=-1), dict(k_stride=(0, 0, 63)), dict(v_stride=(64, 64, 8))):
            assert call(p=_params(**bad)) == INVALID, bad
        for bad in (dict(d=32), dict(block=32), dict(L=65537)):
            assert call(p=_params(**bad)) == UNSUPPORTED, bad
        if fn is L.asa_cache_read:
            assert call(p=_params(k_stride=(0, 6400, 64))) == call(p=_params(v_stride=(12800, 64, 64))) == INVALID
        odd = ctypes.c_void_p(0x10008)
        assert call(k=odd) == call(v=odd) == call(s=ctypes.c_void_p(0x10001)) == call(n=ctypes.c_void_p(0x10002)) == INVALID


def test_cached_attention_refusals():
    L = binding.load()

    def call(p=_params(), c=_cache(), length=FAKE, q=FAKE, ptr=None, idx=None, o=FAKE, lse=FAKE, w=FAKE, size=1 << 40):
        return L.asa_attn_cache(p, c, length, q, ptr, idx, o, lse, w, size, None)

    ws = L.asa_attn_cache_workspace_bytes
    assert call(p=_params(o_stride=(0, 6400, 64))) == call(p=_params(o_stride=(25600, 32, 64))) == INVALID
    assert ws(_params(L=1), _cache(max_blocks=1000)) > 0
    for args in (dict(p=None), dict(c=None), dict(length=None), dict(q=None), dict(o=None), dict(lse=None), dict(ptr=FAKE), dict(idx=FAKE),
                 dict(q=ctypes.c_void_p(0x10008)), dict(o=ctypes.c_void_p(0x10004)), dict(lse=ctypes.c_void_p(0x10002)),
                 dict(length=ctypes.c_void_p(0x10001))):
        assert call(**args) == INVALID, args
    for bad in (dict(H_kv=3), dict(H_kv=8), dict(H_kv=0), dict(max_blocks=0)):
        assert call(c=_cache(**bad)) == INVALID and ws(_params(), _cache(**bad)) == 0, bad
    for bad in (dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(L=0), dict(q_stride=(0, 0, 8)), dict(o_stride=(4, 8, 64))):
        assert call(p=_params(**bad)) == INVALID and ws(_params(**bad), _cache()) == 0, bad
    assert call(p=_params(d=256)) == UNSUPPORTED and call(c=_cache(max_blocks=70000)) == UNSUPPORTED
    need = ws(_params(L=1), _cache(max_blocks=1000))
    assert call(p=_params(L=1), c=_cache(max_blocks=1000), size=need - 1) == WORKSPACE
    assert call(p=_params(L=1), c=_cache(max_blocks=1000), w=None) == WORKSPACE


def test_the_binding_refuses_host_tensors_and_unknown_words():
    p = binding.Params(B=1, H=2, L=4, d=64, block=64)
    q = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(binding.AsaError, match="device tensors"):
        binding.asa_qk_norm_rope(p, binding.QkNorm(), q, q, q, q)
    c = binding.alloc_kv_cache(1, 2, 1, 64, 64, device="cpu")
    assert c.k.shape == (1, 2, 1, 2, 4, 32, 16) and c.v.shape == (1, 2, 1, 2, 2, 2, 32, 16)
    with pytest.raises(binding.AsaError, match="device tensors"):
        binding.asa_cache_write(p, c, q, q)
    with pytest.raises(binding.AsaError, match="device tensors"):
        binding.asa_attn_cache(p, c, None, q, None, None, q, None, None)
    with pytest.raises(binding.AsaError, match="kind"):
        binding.QkNorm(kind="batch").c(p, 0)
    with pytest.raises(binding.AsaError, match="pairing"):
        binding.QkNorm(pairing="thirds").c(p, 0)
    with pytest.raises(binding.AsaError, match="cos, sin"):
        binding.QkNorm(rot_dim=64, cos=torch.zeros(3, 16), sin=torch.zeros(3, 16)).c(p, 0)
    with pytest.raises(binding.AsaError, match="strides"):
        binding._rows(q.transpose(1, 2).contiguous().transpose(1, 2), "q", (1, 2, 4, 64), (0, 0, 0), -1)
    with pytest.raises(binding.AsaError, match="expected"):
        binding._rows(q.float(), "q", (1, 2, 4, 64), (0, 0, 0), -1)
    with pytest.raises(binding.AsaError, match="expected"):
        binding._flat(torch.zeros(3, dtype=torch.int64), "length", torch.int32, 3, -1)
    with pytest.raises(binding.AsaError, match="codes expected"):
        c.c(binding.Params(B=1, H=2, L=4, d=128, block=64), -1)


def test_the_oracles_codes_are_those_of_e4m3():
    """Every code's value, and rounding of values between all neighbours, against torch's conversion."""
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(codes.view(torch.float8_e4m3fn).double().numpy(), ref.VALUES, equal_nan=True)
    v = np.sort(ref.VALUES[np.isfinite(ref.VALUES)])
    mid = (v[:-1] + v[1:]) / 2
    x = np.unique(np.concatenate([v, mid, np.nextafter(mid, np.inf).astype(np.float32), (mid * (1 + 1e-6)), (mid * (1 - 1e-6))])).astype(np.float32)
    x = x[np.abs(x) <= 448]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.VALUES[ref.encode(x)], want)


def test_the_oracles_scale_is_the_least_that_holds():
    for a in (0.0, 1e-39, 1.0, 447.9, 448.0, 448.1, 449.0, 895.9, 896.0, 3.38e38, 2.0 ** -95):
        s = ref.scale_for(a)
        assert a <= 448 * s and (s == 2.0 ** ref.LEAST_EXP or a > 448 * s / 2)


def test_the_oracles_attention_on_plain_values():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((1, 2, n, 8)) for n in (3, 10, 10))
    o, lse, _, _ = ref.attention(q, k, v, [10], 4, 0.5)
    s = q @ k.transpose(0, 1, 3, 2) * 0.5
    p = np.exp(s)
    assert np.allclose(o, p / p.sum(-1, keepdims=True) @ v) and np.allclose(lse, np.log(p.sum(-1)))
    o2, *_ = ref.attention(q, k, v, [10], 4, 0.5, [[[[0, 1, 2]], [[2, 0, 1]]]])
    assert np.allclose(o, o2)
    o3, lse3, _, _ = ref.attention(q, k, v, [0], 4, 0.5)
    assert (o3 == 0).all() and np.isneginf(lse3).all()
