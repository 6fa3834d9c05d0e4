"""A tensor that a call may do without: its strides in the parameters have no say where it is absent."""

import pytest
import torch

from paper_2508_10774_amd import binding as asa

pytestmark = pytest.mark.gpu
# overlapping rows, strides that no row of 16-byte pieces has, fewer than a row's channels apart, negative
STRIDES = [(0, 0, 64), (64, 64, 8), (100, 50, 65), (-64, 64, 64)]


@pytest.mark.parametrize("strides", STRIDES)
def test_queries_alone(strides):
    g = torch.Generator(device="cuda").manual_seed(1)
    q, gq = (torch.randn(2, 3, 40, 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    n = asa.QkNorm(H_kv=2)
    plain = asa.Params(B=2, H=3, L=40, d=64, block=64)

    def both(p, n):
        ws = asa.alloc_workspace(asa.asa_qk_norm_rope_bwd_workspace_bytes(p, n))
        out, dq, dw = torch.empty_like(q), torch.empty_like(q), torch.empty(64, device="cuda")
        asa.asa_qk_norm_rope(p, n, q, None, out, None)
        asa.asa_qk_norm_rope_bwd(p, n, q, None, gq, None, dq, None, dw, None, None, None, ws)
        return out, dq, dw

    want = both(plain, n)
    got = both(asa.Params(B=2, H=3, L=40, d=64, block=64, k_stride=strides), asa.QkNorm(H_kv=2, k_out_stride=strides))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("strides", STRIDES)
@pytest.mark.parametrize("there", ["k", "v"])
def test_one_of_keys_and_values(strides, there):
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(2, 3, 70, 64, generator=g, device="cuda").to(torch.bfloat16)
    caches = [asa.alloc_kv_cache(2, 3, 2, 64, 64) for _ in range(2)]
    other = "v_stride" if there == "k" else "k_stride"
    out = []
    for cache, more in zip(caches, ({}, {other: strides})):
        p = asa.Params(B=2, H=3, L=70, d=64, block=64, **more)
        back = torch.zeros_like(x)
        asa.asa_cache_write(p, cache, x if there == "k" else None, x if there == "v" else None)
        asa.asa_cache_read(p, cache, back if there == "k" else None, back if there == "v" else None)
        out.append(back)
    assert torch.equal(*out) and (out[0] != 0).any()
    assert all(torch.equal(getattr(caches[0], n), getattr(caches[1], n)) for n in ("k", "v", "k_scale", "v_scale"))
