"""A row of the cached attention has the same bits whatever the other rows of the call hold."""

import pytest
import torch

from paper_2508_10774_amd import binding as asa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,block", [(64, 64), (128, 128)])
@pytest.mark.parametrize("H,L", [(8, 1), (20, 2), (1, 100), (2, 300)])
def test_a_row_does_not_depend_on_its_neighbours(d, block, H, L):
    """Keys whose scores grow along the sequence, for most queries by little and for one by so much that its sums are brought
    down again and again; that one is then replaced by a query of zeros."""
    blocks = 6
    n = blocks * block
    cache = asa.alloc_kv_cache(1, 1, blocks, d, block)
    g = torch.Generator(device="cuda").manual_seed(3)
    ramp = torch.linspace(0, 1, n, device="cuda")[None, None, :, None]
    k = (ramp + 0.05 * torch.randn(1, 1, n, d, generator=g, device="cuda")).to(torch.bfloat16)
    v = torch.randn(1, 1, n, d, generator=g, device="cuda").to(torch.bfloat16)
    asa.asa_cache_write(asa.Params(B=1, H=1, L=n, d=d, block=block), cache, k, v)
    length = torch.tensor([n - 7], dtype=torch.int32, device="cuda")
    # scores reach 5 log2 units at most, less than the 2^8 that a row's own maximum may lag by
    q = torch.rand(1, H, L, d, generator=g, device="cuda") * (3.0 / d ** 0.5)
    p = asa.Params(B=1, H=H, L=L, d=d, block=block)
    ws = asa.alloc_workspace(asa.asa_attn_cache_workspace_bytes(p, cache))

    def run(odd):
        x = q.clone().reshape(H * L, d)
        x[H * L // 2] = odd
        x = x.reshape(q.shape).to(torch.bfloat16)
        o, lse = torch.empty_like(x), torch.empty(H, L, device="cuda")
        asa.asa_attn_cache(p, cache, length, x, None, None, o, lse, ws)
        torch.cuda.synchronize()
        return o.reshape(H * L, d), lse.reshape(H * L)

    (o, lse), (o2, lse2) = run(30.0), run(0.0)
    others = [r for r in range(H * L) if r != H * L // 2]
    assert not torch.equal(o[H * L // 2], o2[H * L // 2])
    assert torch.equal(o[others], o2[others]) and torch.equal(lse[others], lse2[others])
