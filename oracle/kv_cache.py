"""Plain 64-bit implementations of the operators around the attention call (test infrastructure only).

Norm and rotation of queries and keys with their gradients, the 8-bit cache of keys and values, attention over it:
written from the formulas in ``include/asa.h``, element by element where that is the definition.
"""

import numpy as np

LEAST_EXP, MOST_EXP, LARGEST = -100, 120, 448.0


# ------------------------------------------------------------------------------ norm and rotation

def _pairs(rot, pairing):
    t = np.arange(rot // 2)
    return (2 * t, 2 * t + 1) if pairing == "adjacent" else (t, t + rot // 2)


def angles(cos, sin, B, L, first_row, start):
    """cos and sin [B, L, pairs] of the call's tokens; rows outside the table turn nothing."""
    c, s = np.ones((B, L, cos.shape[1])), np.zeros((B, L, cos.shape[1]))
    for b in range(B):
        for l in range(L):
            row = first_row + l + (0 if start is None else int(start[b]))
            if 0 <= row < cos.shape[0]:
                c[b, l], s[b, l] = cos[row], sin[row]
    return c, s


def turn(x, c, s, pairing):
    """x [B, n, L, d], c and s [B, L, pairs]."""
    y = x.copy()
    a, b = _pairs(2 * c.shape[-1], pairing)
    c, s = c[:, None], s[:, None]
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def normed(x, kind, eps):
    """(normalised x, 1 / deviation)"""
    x = x - x.mean(-1, keepdims=True) if kind == "layer" else x
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def norm_rope(x, w, b, kind, eps, c=None, s=None, pairing="adjacent"):
    z = normed(x, kind, eps)[0] * w + b
    return z if c is None else turn(z, c, s, pairing)


def norm_rope_bwd(x, dy, w, kind, eps, c=None, s=None, pairing="adjacent"):
    """dx, dw, db and the sums of the absolute terms of dw and db."""
    dz = dy if c is None else turn(dy, c, -s, pairing)
    xh, r = normed(x, kind, eps)
    gw = dz * w
    dx = gw - xh * (gw * xh).mean(-1, keepdims=True)
    if kind == "layer":
        dx = dx - gw.mean(-1, keepdims=True)
    ax = (0, 1, 2)
    return dx * r, (dz * xh).sum(ax), dz.sum(ax), np.abs(dz * xh).sum(ax), np.abs(dz).sum(ax)


# ------------------------------------------------------------------------------ 8-bit codes

def code_values():
    """Value of each of the 256 codes: sign, 4 bits of exponent (bias 7), 3 of fraction; no infinity."""
    out = np.empty(256)
    for code in range(256):
        e, f = code >> 3 & 15, code & 7
        x = np.nan if (e, f) == (15, 7) else f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        out[code] = -x if code & 128 else x
    return out


VALUES = code_values()
_POSITIVE = VALUES[:127]          # ascending


def encode(x):
    """Codes of the nearest values, ties to the even code; what is not finite becomes NaN (0x7f)."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    a = np.minimum(np.abs(np.where(finite, x, 0.0)), LARGEST)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dlo, dhi = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((dlo < dhi) | ((dlo == dhi) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    code = code | np.where(np.signbit(x), 128, 0).astype(np.uint8)
    return np.where(finite, code, np.uint8(0x7F))


def scale_for(absmax):
    """The least 2^e, e in [LEAST_EXP, MOST_EXP], with absmax <= 448 * 2^e."""
    for e in range(LEAST_EXP, MOST_EXP):
        if absmax <= LARGEST * 2.0 ** e:
            return 2.0 ** e
    return 2.0 ** MOST_EXP


class Cache:
    """codes[name] [B, H, blocks, block, d] in plain order, scale[name] [B, H, blocks]."""

    def __init__(self, B, H, blocks, block, d):
        self.block, self.blocks = block, blocks
        self.codes = {n: np.zeros((B, H, blocks, block, d), np.uint8) for n in "kv"}
        self.scale = {n: np.full((B, H, blocks), 2.0 ** LEAST_EXP) for n in "kv"}

    def write(self, name, x, start, count):
        B, H, L, _ = x.shape
        codes, scale = self.codes[name], self.scale[name]
        for b in range(B):
            if start[b] < 0:
                continue
            end = min(start[b] + min(max(count[b], 0), L), self.blocks * self.block)
            for j in range(self.blocks):
                lo, hi = max(start[b] - j * self.block, 0), min(end - j * self.block, self.block)
                if lo >= hi:
                    continue
                for h in range(H):
                    new = x[b, h, j * self.block + lo - start[b]:j * self.block + hi - start[b]]
                    absmax = np.abs(new[np.isfinite(new)]).max(initial=0.0)
                    s, old = scale_for(absmax), scale[b, h, j]
                    if lo > 0 and old > s:
                        s = old
                    if lo > 0 and s != old:
                        held = (VALUES[codes[b, h, j, :lo]] * old).astype(np.float32).astype(np.float64)
                        codes[b, h, j, :lo] = encode((held / s).astype(np.float32))
                    codes[b, h, j, lo:hi] = encode((new / s).astype(np.float32))
                    scale[b, h, j] = s

    def values(self, name):
        """[B, H, blocks * block, d]"""
        x = VALUES[self.codes[name]] * self.scale[name][..., None, None]
        return x.reshape(*x.shape[:2], -1, x.shape[-1])


def k_layout(codes):
    """[.., block, d] -> [.., block/32, d/16, 32, 16], by the definition."""
    *lead, n, d = codes.shape
    out = np.empty((*lead, n // 32, d // 16, 32, 16), codes.dtype)
    for t in range(n):
        for x in range(d):
            out[..., t // 32, x // 16, t % 32, x % 16] = codes[..., t, x]
    return out


def v_layout(codes):
    """[.., block, d] -> [.., block/32, d/32, 2, 32, 16]: token 8 m + 4 h + j at [h][channel][4 m + j]."""
    *lead, n, d = codes.shape
    out = np.empty((*lead, n // 32, d // 32, 2, 32, 16), codes.dtype)
    for t in range(n):
        m, h, j = t % 32 // 8, t % 8 // 4, t % 4
        for x in range(d):
            out[..., t // 32, x // 32, h, x % 32, 4 * m + j] = codes[..., t, x]
    return out


# ------------------------------------------------------------------------------ attention

def attention(q, k, v, length, block, scale, lists=None):
    """q [B, H, L, d], k and v [B, H_kv, tokens, d] -> o, lse [B, H, L], sum of p |v|, and the largest sum of
    |q_i k_i| * scale of each row.  lists[b][h_kv][query block]: kept blocks."""
    B, H, L, d = q.shape
    H_kv = k.shape[1]
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, terms = np.full((B, H, L), -np.inf), np.zeros((B, H, L))
    for b in range(B):
        n = min(max(int(length[b]), 0), k.shape[2])
        for h in range(H):
            g = h // (H // H_kv)
            for i in range(-(-L // block)):
                rows = slice(i * block, min((i + 1) * block, L))
                at = np.arange(n)
                if lists is not None:
                    kept = [j for j in lists[b][g][i] if j >= 0]
                    at = np.concatenate([np.arange(j * block, (j + 1) * block) for j in kept] + [np.empty(0, int)])
                    at = at[at < n].astype(int)
                if not len(at):
                    continue
                s = q[b, h, rows] @ k[b, g, at].T * scale
                m = s.max(-1, keepdims=True)
                p = np.exp(s - m)
                total = p.sum(-1, keepdims=True)
                o[b, h, rows] = p / total @ v[b, g, at]
                mag[b, h, rows] = p / total @ np.abs(v[b, g, at])
                lse[b, h, rows] = (m + np.log(total))[:, 0]
                terms[b, h, rows] = (np.abs(q[b, h, rows]) @ np.abs(k[b, g, at]).T).max(-1) * scale
    return o, lse, mag, terms
