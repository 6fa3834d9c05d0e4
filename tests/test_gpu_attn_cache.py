"""Attention over the 8-bit cache against 64 bits.

Tolerances.  Codes are widened exactly.  A score is an fp32 sum of d products: off by at most d * 2^-24 of the sum of their
magnitudes (terms), by the factor and the maximum taken off a few 2^-24 of it more: 2^-16 * terms in all, which is also the
relative error that a probability gets from it; the exponential adds 2^-20.  Probabilities are rounded to bf16 (2^-8) before
the second product, the result is rounded to bf16 (2^-8).  Sums of n keys in fp32, in parts: n / 8 * 2^-24 < 2^-12 here.
"""

import numpy as np
import pytest
import torch

from oracle import kv_cache as ref
from paper_2508_10774_amd import binding as asa

pytestmark = pytest.mark.gpu


def _np(t):
    return t.double().cpu().numpy()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Held:
    """A cache with `tokens` written to every sequence, and the values it stands for."""

    def __init__(self, seed, B, H, blocks, d, block, tokens):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.B, self.H, self.blocks, self.d, self.block = B, H, blocks, d, block
        self.cache = asa.alloc_kv_cache(B, H, blocks, d, block)
        gain = torch.exp(torch.randn(2, B, H, 1, 1, generator=g, device="cuda"))
        x = (torch.randn(2, B, H, tokens, d, generator=g, device="cuda") * gain).to(torch.bfloat16)
        asa.asa_cache_write(asa.Params(B=B, H=H, L=tokens, d=d, block=block), self.cache, x[0], x[1])
        self.read()

    def read(self):
        n = self.blocks * self.block
        out = [torch.zeros(self.B, self.H, n, self.d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        asa.asa_cache_read(asa.Params(B=self.B, H=self.H, L=n, d=self.d, block=self.block), self.cache, *out)
        self.k, self.v = (_np(t) for t in out)


def _lists(mask, junk=0):
    """row_ptr, col_idx of a [B, H_kv, rows, blocks] bool mask, entries in a shuffled order; behind them junk."""
    B, H, rows, blocks = mask.shape
    rng = np.random.default_rng(3)
    ptr, idx = np.zeros((B * H, rows + 1), np.int32), np.full((B * H, rows * blocks), junk, np.int32)
    kept = [[[list(rng.permutation(np.nonzero(mask[b, h, i])[0])) for i in range(rows)] for h in range(H)] for b in range(B)]
    for b in range(B):
        for h in range(H):
            s, n = b * H + h, 0
            for i in range(rows):
                idx[s, n:n + len(kept[b][h][i])] = kept[b][h][i]
                n += len(kept[b][h][i])
                ptr[s, i + 1] = n
    return _i32(ptr.tolist()), _i32(idx.tolist()), kept


def _run(h, q, length, lists=(None, None), o=None, scale=0.0):
    B, H, L, d = q.shape
    o = torch.full((B, H, L, d), float("nan"), dtype=torch.bfloat16, device="cuda") if o is None else o
    lse = torch.full((B * H, L), float("nan"), device="cuda")
    p = asa.Params(B=B, H=H, L=L, d=d, block=h.block, scale=scale, q_stride=q.stride()[:3], o_stride=o.stride()[:3])
    ws = asa.alloc_workspace(asa.asa_attn_cache_workspace_bytes(p, h.cache))
    ws.fill_(255)                                        # NaN where nothing is written
    asa.asa_attn_cache(p, h.cache, length, q, *lists, o, lse, ws)
    torch.cuda.synchronize()
    return o, lse


def _check(h, q, length, got, kept=None, scale=None):
    o, lse = _np(got[0]), _np(got[1]).reshape(q.shape[:3])
    B, H, L, d = q.shape
    want, want_lse, mag, terms = ref.attention(_np(q), h.k, h.v, length, h.block, scale or d ** -0.5, kept)
    none = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(lse), none)
    assert (o[none] == 0).all()
    slack = 2.0 ** -16 * terms[..., None]
    allow = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12 + 2 * slack + 2.0 ** -20) * mag
    err = np.abs(o - want)
    assert (err <= allow + 1e-30).all(), (err / (allow + 1e-30)).max()
    ok = ~none
    allow = 2.0 ** -12 * 2.0 ** -8 + slack[..., 0] + 2.0 ** -20 * np.abs(np.where(ok, want_lse, 0))
    assert (np.abs(lse[ok] - want_lse[ok]) <= allow[ok]).all(), (np.abs(lse[ok] - want_lse[ok]) / allow[ok]).max()


def _q(seed, B, H, L, d, packed=False, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(B, L, H, d, generator=g, device="cuda") * gain).to(torch.bfloat16).transpose(1, 2)
    return x if packed else x.contiguous()


@pytest.mark.parametrize("d,block", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("H,Hkv,L", [(2, 2, 1), (8, 2, 1), (3, 1, 5), (2, 2, 31), (2, 1, 33), (1, 1, 64), (4, 2, 100), (2, 2, 300), (40, 1, 1)])
def test_every_block(d, block, H, Hkv, L):
    """Lengths from nothing to all of it, with junk (NaN codes among it) behind them."""
    h = Held(1, 4, Hkv, 5, d, block, 5 * block)
    n = 5 * block
    length = [0, 1, block + 37, n]
    for b in range(4):                                   # NaN codes at and past each length
        for name, lay in (("k", ref.k_layout), ("v", ref.v_layout)):
            at = lay((np.arange(n).reshape(1, 5, block, 1) >= length[b]) & np.ones((1, 1, 1, d), bool))[0]
            codes = getattr(h.cache, name)[b]
            codes[:, torch.from_numpy(at).cuda()] = 0x7F
    q = _q(2, 4, H, L, d, packed=L % 2 == 1)
    got = _run(h, q, _i32(length))
    _check(h, q, length, got)


@pytest.mark.parametrize("d,block", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("H,Hkv,L", [(2, 2, 1), (6, 2, 3), (2, 2, 70), (4, 2, 333)])
def test_lists(d, block, H, Hkv, L):
    """Shuffled lists, rows without a block, blocks past a sequence's end, entries that are no block."""
    B, blocks = 3, 6
    h = Held(4, B, Hkv, blocks, d, block, blocks * block)
    rows = -(-L // block)
    mask = np.random.default_rng(7).random((B, Hkv, rows, blocks)) < 0.5
    mask[0, 0, 0] = False
    mask[1, :, -1] = [False] * (blocks - 1) + [True]      # a block that the sequence does not reach
    ptr, idx, kept = _lists(mask, junk=10 ** 9)
    length = [blocks * block, 3 * block + 5, 2 * block]
    q = _q(5, B, H, L, d)
    got = _run(h, q, _i32(length), (ptr, idx))
    _check(h, q, length, got, kept)
    bad = idx.clone()                                    # negative and far entries are skipped
    bad[0, :1] = -5
    bad[2, :1] = 2 ** 30
    kept[0] = [[list(r) for r in s] for s in kept[0]]
    first = {0: -5, 2: 2 ** 30}
    for s, x in first.items():
        b, hk = divmod(s, Hkv)
        for i in range(rows):
            if kept[b][hk][i]:
                kept[b][hk][i] = [x if x < 0 else -1] + kept[b][hk][i][1:]
                break
    if ptr[0, -1] > 0 and ptr[2, -1] > 0:
        _check(h, q, length, _run(h, q, _i32(length), (ptr, bad)), kept)


def test_one_token_on_long_sequences_is_split():
    """Few rows and many blocks: the keys are shared out and joined; large scores, a head whose maximum comes last."""
    h = Held(8, 2, 2, 90, 64, 128, 90 * 128)
    q = _q(9, 2, 4, 1, 64, gain=4.0)
    length = [90 * 128, 5 * 128 + 1]
    assert asa.asa_attn_cache_workspace_bytes(asa.Params(B=2, H=4, L=1, d=64, block=128), h.cache) > 0
    got = _run(h, q, _i32(length))
    _check(h, q, length, got)
    again = _run(h, q, _i32(length))
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("H,L,d,block,blocks,parts", [(12, 400, 64, 128, 40, (5, 64)), (12, 400, 128, 64, 70, (5, 64)),
                                                      (18, 1500, 128, 128, 32, (2, 4)), (66, 1000, 64, 64, 30, (2, 4))])
def test_many_rows_in_parts(H, L, d, block, blocks, parts):
    """Thousands of rows whose keys are cut into a few parts, and into more than are joined at once; a sequence too short for
    most of the parts; NaN in the workspace."""
    h = Held(20, 2, H, blocks, d, block, blocks * block)
    p = asa.Params(B=2, H=H, L=L, d=d, block=block)
    rows = 2 * H * -(-L // block) * block
    assert rows > 4096
    cut = asa.asa_attn_cache_workspace_bytes(p, h.cache) // (rows * (d + 2) * 4)
    assert parts[0] <= cut <= parts[1], cut
    q = _q(21, 2, H, L, d, packed=True, gain=2.0)
    length = [blocks * block - 3, 70]
    o, lse = _run(h, q, _i32(length))
    k, v = h.k, h.v
    for head in (0, H // 2, H - 1):
        one = slice(head, head + 1)
        h.k, h.v = k[:, one], v[:, one]
        _check(h, q[:, one], length, (o[:, one], lse.reshape(2, H, L)[:, one]))


def test_strided_output_scale_and_canaries():
    h = Held(10, 2, 2, 3, 128, 64, 150)
    q = _q(11, 2, 4, 77, 128, packed=True)
    base = torch.full((2, 78, 5, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    o = base[:, :77, :4].transpose(1, 2)
    got = _run(h, q, _i32([150, 64]), o=o, scale=0.3)
    _check(h, q, [150, 64], got, scale=0.3)
    assert (base[:, 77] == 7).all() and (base[:, :, 4] == 7).all()


def test_scales_of_any_size():
    """Scales that are no powers of two, very small and very large ones: S and O by the value they stand for."""
    h = Held(12, 1, 1, 4, 64, 64, 256)
    h.cache.k_scale.copy_(torch.tensor([0.013, 3e-30, 0.02, 1e-4], device="cuda"))
    h.cache.v_scale.copy_(torch.tensor([0.3, 1e-20, 1e20, 0.77], device="cuda"))
    cv = {n: ref.VALUES[getattr(h.cache, n).cpu().numpy()] for n in "kv"}
    k = cv["k"].transpose(0, 1, 2, 3, 5, 4, 6).reshape(1, 1, 4, 64, 64)
    v = cv["v"].reshape(1, 1, 4, 2, 2, 2, 32, 4, 4).transpose(0, 1, 2, 3, 7, 5, 8, 4, 6).reshape(1, 1, 4, 64, 64)
    h.k = (k * _np(h.cache.k_scale)[..., None, None]).reshape(1, 1, 256, 64)
    h.v = (v * _np(h.cache.v_scale)[..., None, None]).reshape(1, 1, 256, 64)
    for L in (1, 40, 200):
        for lists in (None, [0, 1, 3], [2], [1]):
            q = _q(13, 1, 1, L, 64)
            rows = -(-L // 64)
            ptr = idx = kept = None
            if lists is not None:
                mask = np.zeros((1, 1, rows, 4), bool)
                mask[..., lists] = True
                ptr, idx, kept = _lists(mask)
            _check(h, q, [256], _run(h, q, _i32([256]), (ptr, idx)), kept)


@pytest.mark.parametrize("span", [6.0, 40.0, 300.0])
@pytest.mark.parametrize("falling", [False, True])
def test_rising_and_falling_scores(span, falling):
    """Scores that grow from key to key by little and by much (the running maximum is brought up late), or fall."""
    h = Held(22, 1, 1, 6, 64, 64, 384)
    ramp = torch.linspace(-1, 1, 384, device="cuda")
    ramp = (ramp.flip(0) if falling else ramp)[None, None, :, None]
    g = torch.Generator(device="cuda").manual_seed(23)
    k = (ramp + 0.01 * torch.randn(1, 1, 384, 64, generator=g, device="cuda")).to(torch.bfloat16)
    asa.asa_cache_write(asa.Params(B=1, H=1, L=384, d=64, block=64), h.cache, k, None)
    h.read()
    for L in (1, 40, 100):
        q = torch.full((1, 1, L, 64), span / 8, device="cuda") * torch.linspace(0.2, 1, L, device="cuda")[:, None]
        q = q.to(torch.bfloat16)
        _check(h, q, [384], _run(h, q, _i32([384])))


def test_blocks_of_scale_zero_and_many_short_sequences():
    """A block of zeros at a scale of 0 weighs in like any other; more (sequence, head) pairs than a grid axis holds."""
    h = Held(16, 1, 1, 3, 64, 64, 192)
    h.cache.k_scale[0, 0, 1] = 0.0
    h.cache.v_scale[0, 0, 1] = 0.0
    h.read()
    for L in (1, 70):
        q = _q(17, 1, 1, L, 64)
        _check(h, q, [192], _run(h, q, _i32([192])))
    B, H = 17000, 4
    h = Held(18, B, 1, 1, 64, 64, 3)
    q = _q(19, B, H, 1, 64)
    o, lse = _run(h, q, torch.full((B,), 3, dtype=torch.int32, device="cuda"))
    k, v = (torch.from_numpy(x).cuda()[:, :, :3] for x in (h.k, h.v))
    s = torch.matmul(q.double(), k.transpose(-1, -2).contiguous()) / 8
    want = torch.matmul(torch.softmax(s, -1), v)
    # 2^-8 of the result and 2^-8 of sum p |v|, which is at most the largest |v|
    allow = 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * v.abs().amax(2, keepdim=True)
    assert ((o.double() - want).abs() <= allow).all()
    assert (lse.reshape(B, H, 1).double() - torch.logsumexp(s, -1)).abs().max() <= 1e-4
    n = asa.QkNorm(H_kv=H)
    p = asa.Params(B=B, H=H, L=1, d=64, block=64)
    out = [torch.empty_like(q) for _ in range(2)]
    asa.asa_qk_norm_rope(p, n, q, q, *out)
    want = q.double() / (q.double().square().mean(-1, keepdim=True) + 1e-6).sqrt()
    assert torch.equal(out[0], out[1]) and ((out[0].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True)).all()


def test_values_that_are_not_finite():
    """NaN among the keys a row sees makes that row NaN, and no row that does not see it."""
    h = Held(14, 1, 2, 4, 64, 64, 256)
    h.cache.k[0, 0, 1, 0, 0, 5, 3] = 0x7F
    mask = np.ones((1, 2, 3, 4), bool)
    mask[0, 0, 1, 1] = False
    ptr, idx, kept = _lists(mask)
    q = _q(15, 1, 2, 192, 64)
    o, lse = _run(h, q, _i32([256]), (ptr, idx))
    seen = torch.isnan(o.float()).all(-1)
    assert seen[0, 0, :64].all() and seen[0, 0, 128:].all() and not seen[0, 0, 64:128].any() and not seen[0, 1].any()
    assert torch.equal(torch.isnan(lse.reshape(1, 2, 192)), seen)
    h.read()
    h.k[0, 0, 69] = 0.0
    for r in (slice(64, 128),):
        sub = q[:, :, r]
        want, *_ = ref.attention(_np(sub), h.k, h.v, [256], 64, 64 ** -0.5, [[[kept[0][0][1]], [kept[0][1][1]]]])
        assert np.abs(_np(o[:, :, r]) - want).max() <= 2e-2
