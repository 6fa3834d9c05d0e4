"""Norm of queries and keys with their rotation, and its gradients, against the formulas in 64 bits.

Tolerances.  A result is rounded to bf16 once: 2^-8 of its value.  In front of that everything is fp32: a row's sum of D <=
128 squares is a sum of 8 and then a tree of 4, its relative error below 12 * 2^-24, the reciprocal root halves that and
adds a few 2^-24; with the products and the rotation a value is off by less than 32 * 2^-24 = 2^-19 of the
magnitudes that meet in it.  Those are at most the row's largest |z| twice: 2^-18 of the row's largest.  In LAYER the mean
is taken off first, by values that may be larger than what remains: 2^-18 of (largest |x| * r * largest |weight|) covers it.
Turning back a gradient, a c + b s, may cancel: its error is a few 2^-24 of |a c| + |b s|, not of the result (a single token
whose result is a hundredth of those showed that a bound by the result alone cannot hold), so the gradients'
magnitudes are taken before the two meet.
"""

import numpy as np
import pytest
import torch

from oracle import kv_cache as ref
from paper_2508_10774_amd import binding as asa

pytestmark = pytest.mark.gpu
F32 = 2.0 ** -18


def _np(t):
    return t.detach().double().cpu().numpy()


def _tensors(g, B, counts, L, d, packed):
    x = torch.randn(B, L, sum(counts), d, generator=g, device="cuda") * torch.rand(sum(counts), 1, generator=g, device="cuda").add(0.3)
    if packed:
        x = x.to(torch.bfloat16)
        return [t.transpose(1, 2) for t in x.split(counts, dim=2)]
    return [t.transpose(1, 2).contiguous().to(torch.bfloat16) for t in x.split(counts, dim=2)]


def _like(x, packed):
    B, n, L, d = x.shape
    t = torch.full((B, L, n + 1, d) if packed else (B, n, L, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    return t[:, :, :n].transpose(1, 2) if packed else t


def _case(seed, B, H, Hkv, L, d, kind, pairing, rot, rows=None, first=0, start=None, packed=False, eps=1e-6):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k = _tensors(g, B, [H, Hkv], L, d, packed)
    rows = rows or L
    angle = torch.rand(rows, max(rot // 2, 1), generator=g, device="cuda") * 6.3
    st = torch.tensor(start, dtype=torch.int32, device="cuda") if start is not None else None
    w = [torch.randn(d, generator=g, device="cuda") + 1 for _ in range(2)]
    b = [torch.randn(d, generator=g, device="cuda") if kind == "layer" else None for _ in range(2)]
    gq, gk = _tensors(g, B, [H, Hkv], L, d, False)
    n = asa.QkNorm(H_kv=Hkv, kind=kind, eps=eps, q_weight=w[0], k_weight=w[1], q_bias=b[0], k_bias=b[1], rot_dim=rot,
                   pairing=pairing, cos=angle.cos() if rot else None, sin=angle.sin() if rot else None, first_row=first, start=st)
    p = asa.Params(B=B, H=H, L=L, d=d, block=128, q_stride=q.stride()[:3], k_stride=k.stride()[:3])
    c = s = None
    if rot:
        c, s = ref.angles(_np(n.cos), _np(n.sin), B, L, first, start)
    return p, n, (q, k), (gq, gk), w, b, c, s


def _turned_magnitude(g, c, s, pairing):
    """|a c| + |b s| of each channel that turning back forms."""
    if c is None:
        return np.abs(g)
    return np.maximum(ref.turn(np.abs(g), np.abs(c), np.abs(s), pairing), ref.turn(np.abs(g), np.abs(c), -np.abs(s), pairing))


def _within(got, want, allow):
    ratio = np.abs(got - want) / allow
    assert ratio.max() <= 1.0, (float(ratio.max()), np.unravel_index(np.argmax(ratio), ratio.shape))


def _check_forward(got, x, w, b, n, c, s):
    x, w = _np(x), _np(w)
    b = _np(b) if b is not None else 0.0
    want = ref.norm_rope(x, w, b, n.kind, n.eps, c, s, n.pairing)
    _, r = ref.normed(x, n.kind, n.eps)
    top = np.abs(x).max(-1, keepdims=True) * r * np.abs(w).max() + np.abs(b).max(initial=0) if np.ndim(b) else \
        np.abs(x).max(-1, keepdims=True) * r * np.abs(w).max()
    _within(_np(got), want, 2.0 ** -8 * np.abs(want) + F32 * top)


SHAPES = [
    # B, H, Hkv, L, d, kind, pairing, rot, more
    (1, 1, 1, 1, 64, "rms", "adjacent", 64, {}),
    (3, 2, 2, 1, 128, "rms", "halves", 128, dict(rows=50, start=[0, 49, 7])),
    (2, 5, 3, 37, 128, "layer", "adjacent", 48, dict(first=-5, packed=True)),
    (2, 12, 4, 67, 64, "layer", "halves", 64, dict(rows=40, start=[3, -30])),
    (1, 4, 4, 130, 128, "rms", "halves", 32, dict(packed=True)),
    (1, 9, 1, 333, 64, "rms", "adjacent", 16, dict(packed=True, first=4)),
    (2, 3, 3, 21, 64, "layer", "adjacent", 0, {}),
    (1, 2, 2, 40, 128, "rms", "adjacent", 0, dict(eps=0.0)),
    (1, 6, 2, 19, 64, "layer", "halves", 48, dict(packed=True)),
]


@pytest.mark.parametrize("B,H,Hkv,L,d,kind,pairing,rot,more", SHAPES)
def test_forward(B, H, Hkv, L, d, kind, pairing, rot, more):
    p, n, x, _, w, b, c, s = _case(1, B, H, Hkv, L, d, kind, pairing, rot, **more)
    for strided in (False, True):
        out = [_like(t, strided) for t in x]
        if strided:
            n.q_out_stride, n.k_out_stride = (t.stride()[:3] for t in out)
        asa.asa_qk_norm_rope(p, n, *x, *out)
        torch.cuda.synchronize()
        for i in range(2):
            _check_forward(out[i], x[i], w[i], b[i], n, c, s)
            if strided:          # the head behind the last is not the call's
                base = out[i]._base if out[i]._base is not None else out[i]
                assert torch.isnan(base.reshape(B, L, -1, d)[:, :, -1].float()).all()


@pytest.mark.parametrize("B,H,Hkv,L,d,kind,pairing,rot,more", SHAPES)
def test_backward(B, H, Hkv, L, d, kind, pairing, rot, more):
    p, n, x, gr, w, b, c, s = _case(2, B, H, Hkv, L, d, kind, pairing, rot, **more)
    packed = more.get("packed", False)
    dx = [torch.full((B, L, H + Hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")] if packed else \
        [torch.full_like(t, float("nan")) for t in x]
    if packed:
        dx = [t.transpose(1, 2) for t in dx[0].split([H, Hkv], dim=2)]
    sums = [torch.full((d,), float("nan"), device="cuda") for _ in range(4)]
    ws = asa.alloc_workspace(asa.asa_qk_norm_rope_bwd_workspace_bytes(p, n))
    layer = kind == "layer"
    asa.asa_qk_norm_rope_bwd(p, n, *x, *gr, *dx, sums[0], sums[1], sums[2] if layer else None, sums[3] if layer else None, ws)
    torch.cuda.synchronize()
    for i in range(2):
        want, dw, db, _, _ = ref.norm_rope_bwd(_np(x[i]), _np(gr[i]), _np(w[i]), kind, n.eps, c, s, pairing)
        xh, r = ref.normed(_np(x[i]), kind, n.eps)
        mag = _turned_magnitude(_np(gr[i]), c, s, pairing)
        # the three terms are at most |gw|, |xh| * mean |gw xh| and mean |gw|
        gw = mag * np.abs(_np(w[i]))
        spread = 1 + (np.abs(_np(x[i])).max(-1, keepdims=True) * r if layer else 0)     # of the mean that is taken off
        top = r * (2 * gw.max(-1, keepdims=True) + np.abs(xh) * (gw * np.abs(xh)).mean(-1, keepdims=True)) * spread
        _within(_np(dx[i]), want, 2.0 ** -8 * np.abs(want) + F32 * 2 * top)
        # sums of fp32: fewer than 150 additions in a row here, and 2^-18 of each term
        share = 150 * 2.0 ** -24 + F32
        terms = mag * (np.abs(xh) + (spread - 1))
        _within(_np(sums[i]), dw, share * terms.sum((0, 1, 2)))
        if layer:
            _within(_np(sums[2 + i]), db, share * mag.sum((0, 1, 2)))


def test_gradients_against_differences():
    """The 64-bit formulas themselves: directional derivatives of sum(dy * y) by central differences."""
    rng = np.random.default_rng(5)
    for kind in ("rms", "layer"):
        for pairing in ("adjacent", "halves"):
            x, dy = rng.standard_normal((2, 2, 3, 64)), rng.standard_normal((2, 2, 3, 64))
            w, b = rng.standard_normal(64), rng.standard_normal(64)
            a = rng.uniform(0, 6, (2, 3, 16))
            c, s = np.cos(a), np.sin(a)
            dx, dw, db, _, _ = ref.norm_rope_bwd(x, dy, w, kind, 1e-6, c, s, pairing)
            for arg, grad in ((0, dx), (1, dw), (2, db)):
                u = rng.standard_normal(grad.shape)
                h = 1e-6
                args = [x, w, b]
                f = []
                for sign in (1, -1):
                    moved = list(args)
                    moved[arg] = args[arg] + sign * h * u
                    f.append((dy * ref.norm_rope(*moved, kind, 1e-6, c, s, pairing)).sum())
                assert abs((f[0] - f[1]) / (2 * h) - (grad * u).sum()) <= 1e-6 * max(1.0, abs((grad * u).sum()))


def test_queries_alone_and_in_place():
    p, n, (q, k), (gq, gk), w, b, c, s = _case(3, 2, 3, 2, 45, 128, "layer", "halves", 96)
    both = [torch.empty_like(q), torch.empty_like(k)]
    asa.asa_qk_norm_rope(p, n, q, k, *both)
    alone = torch.empty_like(q)
    asa.asa_qk_norm_rope(p, n, q, None, alone, None)
    qi, ki = q.clone(), k.clone()
    asa.asa_qk_norm_rope(p, n, qi, ki, qi, ki)
    assert torch.equal(alone, both[0]) and torch.equal(qi, both[0]) and torch.equal(ki, both[1])
    ws = asa.alloc_workspace(asa.asa_qk_norm_rope_bwd_workspace_bytes(p, n))
    d = [torch.empty_like(q), torch.empty_like(k)]
    sums = [torch.empty(128, device="cuda") for _ in range(4)]
    asa.asa_qk_norm_rope_bwd(p, n, q, k, gq, gk, *d, *sums, ws)
    again = [torch.zeros(128, device="cuda") for _ in range(4)]
    for place in (0, 1):                                   # dq in the place of q, of dq_out
        ins = [q.clone(), k.clone(), gq.clone(), gk.clone()]
        asa.asa_qk_norm_rope_bwd(p, n, *ins, ins[2 * place], ins[2 * place + 1], *again, ws)
        assert torch.equal(ins[2 * place], d[0]) and torch.equal(ins[2 * place + 1], d[1])
        assert all(torch.equal(a, b) for a, b in zip(sums, again))
    only = torch.empty_like(q)
    asa.asa_qk_norm_rope_bwd(p, n, q, None, gq, None, only, None, again[0], None, None, None, ws)
    assert torch.equal(only, d[0]) and torch.equal(again[0], sums[0])


def test_values_that_are_not_finite_stay_in_their_row():
    p, n, (q, k), _, w, b, c, s = _case(4, 1, 2, 2, 20, 64, "rms", "halves", 32, first=-4)
    want = torch.empty_like(q)
    asa.asa_qk_norm_rope(p, n, q, None, want, None)
    q2 = q.clone()
    q2[0, 1, 7, 3] = float("nan")
    q2[0, 0, 9, 60] = float("inf")
    got = torch.empty_like(q)
    asa.asa_qk_norm_rope(p, n, q2, None, got, None)
    assert torch.isnan(got[0, 1, 7].float()).all() and torch.isnan(got[0, 0, 9, 60].float())
    got[0, 1, 7], got[0, 0, 9] = want[0, 1, 7], want[0, 0, 9]
    assert torch.equal(got, want)


def test_many_tokens_repeat_bit_for_bit_and_sum_well():
    """More items than workgroups: every share of the walk, the same bits twice, and the sums against 64 bits."""
    p, n, x, gr, w, b, c, s = _case(6, 1, 8, 8, 9001, 64, "rms", "adjacent", 64, packed=True)
    ws = asa.alloc_workspace(asa.asa_qk_norm_rope_bwd_workspace_bytes(p, n))
    runs = []
    for _ in range(2):
        ws.fill_(255)
        dx = [torch.empty(1, 9001, 8, 64, dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2)]
        q, k = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in x)
        p.q_stride, p.k_stride = q.stride()[:3], k.stride()[:3]
        sums = [torch.empty(64, device="cuda") for _ in range(2)]
        asa.asa_qk_norm_rope_bwd(p, n, q, k, *gr, *dx, *sums, None, None, ws)
        runs.append((dx, sums))
    assert all(torch.equal(a, b) for u, v in zip(*runs) for a, b in zip(u, v))
    for i in range(2):
        want, dw, _, _, _ = ref.norm_rope_bwd(_np(x[i]), _np(gr[i]), _np(w[i]), "rms", n.eps, c, s, "adjacent")
        terms = _turned_magnitude(_np(gr[i]), c, s, "adjacent") * np.abs(ref.normed(_np(x[i]), "rms", n.eps)[0])
        _within(_np(runs[0][1][i]), dw, (300 * 2.0 ** -24 + F32) * terms.sum((0, 1, 2)))
        assert np.abs(_np(runs[0][0][i]) - want).mean() <= 2.0 ** -8 * np.abs(want).mean()
