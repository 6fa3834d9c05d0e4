"""Attention over the 8-bit cache with lists whose blocks are cut into parts: shuffled lists, entries that are no block in the
middle of a part, rows without a block and rows of very different lengths, against 64 bits.  Tolerances as derived in
test_gpu_attn_cache.py (the checks are its)."""

import numpy as np
import pytest
import torch

from paper_2508_10774_amd import binding as asa
from tests.test_gpu_attn_cache import Held, _check, _i32, _lists, _q, _run

pytestmark = pytest.mark.gpu


def _parts(h, q, length, lists):
    """At least how many parts the call with lists cuts its keys into: a workspace one byte too small for n parts is refused (the
    call with a sufficient one only computes)."""
    B, H, L, d = q.shape
    p = asa.Params(B=B, H=H, L=L, d=d, block=h.block, q_stride=q.stride()[:3])
    o, lse = torch.empty(B, H, L, d, dtype=torch.bfloat16, device="cuda"), torch.empty(B * H, L, device="cuda")
    rows = min(L, h.block) * H // h.H
    tile = 32 if rows <= 32 else 64 if rows <= 64 else 128
    units = B * h.H * -(-L // h.block) * -(-rows // tile)
    part = units * min(rows, tile) * (d + 2) * 4
    n = 0
    while n < 64:
        ws = torch.empty(max((n + 1) * part - 1, 16), dtype=torch.uint8, device="cuda")
        try:
            asa.asa_attn_cache(p, h.cache, length, q, *lists, o, lse, ws)
        except asa.AsaError:
            n += 1
            continue
        break
    torch.cuda.synchronize()
    return n


def _mask(rng, B, Hkv, rows, blocks):
    """Lists of every length: nothing, one block, a few, all of them."""
    share = rng.choice([0.0, 0.05, 0.3, 0.9, 1.0], size=(B, Hkv, rows, 1))
    mask = rng.random((B, Hkv, rows, blocks)) < share
    mask[0, 0, 0] = True                                  # a full row; where there are more, beside it one of one block and an empty one
    if rows > 1:
        mask[0, 0, 1] = False
        mask[0, 0, 1, blocks // 2] = True
        mask[0, 0, -1] = False
    if B > 1:
        mask[1, -1, 0] = False
    return mask


CASES = [  # B, H, Hkv, L, d, block, blocks
    (3, 4, 2, 1, 64, 64, 100), (2, 2, 2, 1, 128, 128, 60), (2, 12, 3, 5, 64, 128, 48), (1, 8, 1, 16, 128, 64, 90),
    (2, 2, 2, 50, 128, 64, 80), (1, 3, 3, 200, 64, 128, 64),
    (2, 12, 12, 400, 64, 128, 40), (2, 12, 12, 400, 128, 64, 70),
]


@pytest.mark.parametrize("B,H,Hkv,L,d,block,blocks", CASES)
def test_lists_in_parts(B, H, Hkv, L, d, block, blocks):
    rng = np.random.default_rng(B * H * L + d + blocks)
    h = Held(31, B, Hkv, blocks, d, block, blocks * block)
    rows = -(-L // block)
    ptr, idx, kept = _lists(_mask(rng, B, Hkv, rows, blocks), junk=10 ** 9)
    # a quarter of the entries become ones that name no block: negative, far away, behind the sequence's end
    idx, junk = idx.cpu().numpy(), rng.random(idx.shape) < 0.25
    junk &= np.arange(idx.shape[1])[None] < ptr.cpu().numpy()[:, -1:]
    junk[0, 1:3] = True                                   # (of the full row at least these)
    junk[0, 0] = False
    idx[junk] = rng.choice([-1, -7, 2 ** 30, blocks, 65535], size=int(junk.sum()))
    for s in range(B * Hkv):
        at = 0
        for i in range(rows):
            n = len(kept[s // Hkv][s % Hkv][i])
            kept[s // Hkv][s % Hkv][i] = [int(j) if 0 <= j < blocks else -1 for j in idx[s, at:at + n]]
            at += n
    lists = ptr, _i32(idx.tolist())
    length = [blocks * block - 3, 70, blocks * block][:B]
    q = _q(32, B, H, L, d, packed=L % 2 == 1, gain=2.0)
    assert _parts(h, q, _i32(length), lists) > 1
    o, lse = _run(h, q, _i32(length), lists)
    again = _run(h, q, _i32(length), lists)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
    if H <= 4:
        _check(h, q, length, (o, lse), kept)
        return
    k, v, group = h.k, h.v, H // Hkv
    for head in sorted({0, group - 1, H // 2, H - 1}):
        one, g = slice(head, head + 1), head // group
        h.k, h.v = k[:, g:g + 1], v[:, g:g + 1]
        _check(h, q[:, one], length, (o[:, one], lse.reshape(B, H, L)[:, one]), [[s[g]] for s in kept])
