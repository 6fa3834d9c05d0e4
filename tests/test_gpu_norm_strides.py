"""The norm's gradients laid out as the caller has them, which need not be as q and k lie: the bits of the call that writes them
in the strides of q and k, and nothing written around them."""

import pytest
import torch

from paper_2508_10774_amd import binding as asa

pytestmark = pytest.mark.gpu


def _heads_between(B, n, L, d):
    """[B, L, n, d] seen as [B, n, L, d]."""
    return torch.full((B, L, n, d), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)


def _within_a_larger(B, n, L, d):
    """Rows of [B + 1, L + 2, n + 1, d + 8]."""
    base = torch.full((B + 1, L + 2, n + 1, d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    return base[:B, :L, :n, :d].transpose(1, 2)


def _packed(B, n, L, d):
    return torch.full((B, n, L, d), 7.0, dtype=torch.bfloat16, device="cuda")


SHAPES = [(1, 1, 1, 1, 64, "rms", "halves"), (2, 5, 3, 37, 128, "layer", "adjacent"), (1, 12, 12, 130, 128, "rms", "adjacent"),
          (3, 4, 1, 1, 64, "layer", "halves"), (1, 9, 1, 333, 64, "rms", "halves"), (1, 1, 1, 50, 128, "rms", "adjacent")]


def _case(B, H, Hkv, L, d, kind, pairing, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(B, L, H + 2 * Hkv, d, generator=g, device="cuda").to(torch.bfloat16)
    q, k, _ = (t.transpose(1, 2) for t in x.split([H, Hkv, Hkv], dim=2))
    gq, gk = (torch.randn(B, n, L, d, generator=g, device="cuda").to(torch.bfloat16) for n in (H, Hkv))
    angle = torch.rand(L, d // 2, generator=g, device="cuda") * 6.3
    n = asa.QkNorm(H_kv=Hkv, kind=kind, q_weight=torch.rand(d, generator=g, device="cuda") + 0.5,
                   k_weight=torch.rand(d, generator=g, device="cuda") + 0.5, rot_dim=d, pairing=pairing, cos=angle.cos(), sin=angle.sin())
    p = asa.Params(B=B, H=H, L=L, d=d, block=128, q_stride=q.stride()[:3], k_stride=k.stride()[:3])
    return p, n, q, k, gq, gk


def _backward(p, n, q, k, gq, gk, dq, dk):
    sums = [torch.full((p.d,), float("nan"), device="cuda") for _ in range(4)]
    ws = asa.alloc_workspace(asa.asa_qk_norm_rope_bwd_workspace_bytes(p, n))
    asa.asa_qk_norm_rope_bwd(p, n, q, k, gq, gk, dq, dk, *sums[:2], *(sums[2:] if n.kind == "layer" else (None, None)), ws)
    torch.cuda.synchronize()
    return dq, dk, *(sums if n.kind == "layer" else sums[:2])


@pytest.mark.parametrize("B,H,Hkv,L,d,kind,pairing", SHAPES)
@pytest.mark.parametrize("lay_q,lay_k", [(_heads_between, _heads_between), (_packed, _heads_between), (_within_a_larger, _packed)])
def test_gradients_laid_out_apart_from_q_and_k(B, H, Hkv, L, d, kind, pairing, lay_q, lay_k):
    p, n, q, k, gq, gk = _case(B, H, Hkv, L, d, kind, pairing)
    as_x = torch.full((B, L, H + 2 * Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    parts = [t.transpose(1, 2) for t in as_x.split([H, Hkv, Hkv], dim=2)]
    want = _backward(p, n, q, k, gq, gk, parts[0], parts[1])
    assert (parts[2] == 7).all()
    got = _backward(p, n, q, k, gq, gk, lay_q(B, H, L, d), lay_k(B, Hkv, L, d))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for t in got[:2]:
        base = t if t._base is None else t._base
        assert (base == 7).sum() >= base.numel() - t.numel()
        rest = base.clone()
        rest.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(7.0)
        assert (rest == 7).all()                          # nothing but the rows is written


def test_rows_of_the_input_that_repeat():
    """One sequence's q and k for every sequence of the batch, gradients for each."""
    p, n, q, k, _, _ = _case(1, 4, 2, 45, 64, "layer", "halves")
    q, k = q.contiguous(), k.contiguous()
    g = torch.Generator(device="cuda").manual_seed(5)
    gq, gk = (torch.randn(3, h, 45, 64, generator=g, device="cuda").to(torch.bfloat16) for h in (4, 2))
    whole = asa.Params(B=3, H=4, L=45, d=64, block=128)
    want = _backward(whole, n, *(t.repeat(3, 1, 1, 1) for t in (q, k)), gq, gk, torch.empty_like(gq), torch.empty_like(gk))
    q3, k3 = q.expand(3, 4, 45, 64), k.expand(3, 2, 45, 64)
    again = asa.Params(B=3, H=4, L=45, d=64, block=128, q_stride=q3.stride()[:3], k_stride=k3.stride()[:3])
    got = _backward(again, n, q3, k3, gq, gk, torch.empty_like(gq), torch.empty_like(gk))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_in_the_place_of_the_incoming_gradients():
    """q and k are slices of a projection; the gradients take the place of those that came in, which are laid out on their own."""
    p, n, q, k, gq, gk = _case(2, 6, 2, 33, 128, "rms", "adjacent")
    want = _backward(p, n, q, k, gq, gk, torch.empty_like(gq), torch.empty_like(gk))
    a, b = gq.clone(), gk.clone()
    got = _backward(p, n, q, k, a, b, a, b)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_rows_that_overlap_are_refused():
    p, n, q, k, gq, gk = _case(2, 3, 3, 20, 64, "rms", "halves")
    dk = torch.empty_like(gk)
    for bad in (torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16, device="cuda").expand(2, 3, 20, 64),
                torch.zeros(1, 3, 20, 64, dtype=torch.bfloat16, device="cuda").expand(2, 3, 20, 64),
                torch.zeros(2, 3, 20, 128, dtype=torch.bfloat16, device="cuda")[..., ::2],
                torch.zeros(2, 3, 20, 68, dtype=torch.bfloat16, device="cuda")[..., :64]):
        with pytest.raises(asa.AsaError):
            _backward(p, n, q, k, gq, gk, bad, dk)
