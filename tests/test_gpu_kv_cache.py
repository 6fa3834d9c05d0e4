"""The 8-bit cache of keys and values: what is written, kept, coded again and read back, bit for bit."""

import numpy as np
import pytest
import torch

from oracle import kv_cache as ref
from paper_2508_10774_amd import binding as asa

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(seed, B, H, L, d, packed, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(B, L, 2 * H, d, generator=g, device="cuda") * gain
    x = x * torch.exp(2 * torch.randn(B, L, 2 * H, 1, generator=g, device="cuda"))        # tokens of very different sizes
    x = x.to(torch.bfloat16)
    k, v = x[:, :, :H].transpose(1, 2), x[:, :, H:].transpose(1, 2)
    return (k, v) if packed else (k.contiguous(), v.contiguous())


def _np(t):
    return t.double().cpu().numpy()


def _write(cache, want, x, block, start, count):
    B, H, L, d = x[0].shape
    p = asa.Params(B=B, H=H, L=L, d=d, block=block, k_stride=x[0].stride()[:3], v_stride=x[1].stride()[:3])
    asa.asa_cache_write(p, cache, *x, start=None if start is None else _i32(start), count=None if count is None else _i32(count))
    for name, t in zip("kv", x):
        want.write(name, _np(t), start or [0] * B, count or [L] * B)


def _same_values(codes, other):
    """Codes equal, NaN by any of its two codes."""
    a, b = np.where(codes & 127 == 127, 127, codes), np.where(other & 127 == 127, 127, other)
    return np.array_equal(a, b)


def _check(cache, want):
    assert np.array_equal(_np(cache.k_scale), want.scale["k"]) and np.array_equal(_np(cache.v_scale), want.scale["v"])
    assert _same_values(cache.k.cpu().numpy(), ref.k_layout(want.codes["k"]))
    assert _same_values(cache.v.cpu().numpy(), ref.v_layout(want.codes["v"]))


@pytest.mark.parametrize("d,block", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("packed", [False, True])
def test_appending_piece_by_piece(d, block, packed):
    """Pieces of all sizes, each sequence at a length of its own, growing and shrinking values."""
    B, H, blocks = 3, 2, 5
    cache, want = asa.alloc_kv_cache(B, H, blocks, d, block), ref.Cache(B, H, blocks, block, d)
    at = [0, 3, block - 1]
    for i, (L, gain) in enumerate([(1, 1.0), (2, 0.01), (29, 30.0), (1, 1e4), (block, 1.0), (block + 35, 0.2), (3, 1e-30)]):
        x = _rows(i, B, H, L, d, packed, gain)
        count = None if i % 2 else [L, max(L - 1, 0), L // 2]
        _write(cache, want, x, block, at, count)
        _check(cache, want)
        at = [a + (L if count is None else c) for a, c in zip(at, count or [L] * B)]


def test_from_an_empty_cache_without_starts():
    cache, want = asa.alloc_kv_cache(2, 3, 3, 64, 64), ref.Cache(2, 3, 3, 64, 64)
    x = _rows(1, 2, 3, 150, 64, True)
    _write(cache, want, x, 64, None, None)
    _check(cache, want)


def test_starts_and_counts_at_their_limits():
    """Before the cache, across its end, past its end, counts out of range, going back into what is held."""
    B, H, blocks, d, block = 6, 1, 3, 64, 64
    cache, want = asa.alloc_kv_cache(B, H, blocks, d, block), ref.Cache(B, H, blocks, block, d)
    x = _rows(1, B, H, 100, d, False)
    _write(cache, want, x, block, [0, 0, 0, 0, 0, 0], None)
    x = _rows(2, B, H, 100, d, False, 3.0)
    _write(cache, want, x, block, [-1, 150, 192, 2 ** 31 - 1, 20, 64], [100, 100, 100, 100, 1000, -5])
    _check(cache, want)


def test_one_tensor_alone():
    cache, want = asa.alloc_kv_cache(1, 2, 2, 128, 128), ref.Cache(1, 2, 2, 128, 128)
    k, v = _rows(3, 1, 2, 130, 128, False)
    p = asa.Params(B=1, H=2, L=130, d=128, block=128)
    asa.asa_cache_write(p, cache, k, None)
    want.write("k", _np(k), [0], [130])
    _check(cache, want)
    asa.asa_cache_write(p, cache, None, v)
    want.write("v", _np(v), [0], [130])
    _check(cache, want)
    out = torch.full_like(v, 7.0)
    asa.asa_cache_read(p, cache, None, out)
    assert np.array_equal(_np(out), want.values("v")[:, :, :130])


def test_values_at_the_borders():
    """Ties, subnormals of the 8-bit type, zeros, the largest and smallest of bf16, NaN and infinities."""
    d, block = 64, 64
    grid = torch.arange(-512, 512, device="cuda").float() / 256                       # ties of every binade
    special = [0.0, -0.0, 448.0, 449.0, 464.0, 480.0, 1e-38, 2.0 ** -133, 3.38e38, -3.38e38, float("nan"), float("inf"), -float("inf"),
               2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9]
    for values in (grid[:512], grid[512:] * 2.0 ** -7, torch.tensor(special[:6] + special[13:], device="cuda"),
                   torch.tensor(special, device="cuda"), torch.zeros(5, device="cuda"), torch.tensor([1e-38, 2.0 ** -133], device="cuda"),
                   torch.full((9,), float("nan"), device="cuda"), torch.full((3,), 3.38e38, device="cuda")):
        x = values.repeat(-(-40 * d // values.numel()))[:40 * d].reshape(1, 1, 40, d).to(torch.bfloat16)
        cache, want = asa.alloc_kv_cache(1, 1, 1, d, block), ref.Cache(1, 1, 1, block, d)
        _write(cache, want, (x, x.flip(2).contiguous()), block, None, None)
        _check(cache, want)
        more = x[:, :, :7].contiguous() * 5
        _write(cache, want, (more, more), block, [40], None)
        _check(cache, want)


def test_a_scale_of_the_users_own():
    """A calibrated scale that is no power of two is kept as long as it is enough, and grown from where it is not."""
    cache, want = asa.alloc_kv_cache(2, 1, 1, 64, 64), ref.Cache(2, 1, 1, 64, 64)
    x = _rows(1, 2, 1, 10, 64, False)
    _write(cache, want, x, 64, None, None)
    own = (torch.rand(2, 1, 1, device="cuda") + 0.3) / 3
    for name in "kv":
        getattr(cache, name + "_scale").copy_(own)
        want.scale[name][:] = _np(own)
    for gain in (1e-3, 1e3):
        x = _rows(2, 2, 1, 9, 64, False, gain)
        p = asa.Params(B=2, H=1, L=9, d=64, block=64)
        asa.asa_cache_write(p, cache, *x, start=_i32([10, 10]))
        for name, t in zip("kv", x):
            t = t.float().cpu().numpy()
            for b in range(2):
                s, old = ref.scale_for(np.abs(t[b]).max()), np.float32(want.scale[name][b, 0, 0])
                s = np.float32(max(s, old))
                if s != old:
                    held = ref.VALUES[want.codes[name][b, 0, 0, :10]].astype(np.float32) * old / s
                    want.codes[name][b, 0, 0, :10] = ref.encode(held)
                want.codes[name][b, 0, 0, 10:19] = ref.encode(t[b, 0] / s)
                want.scale[name][b, 0, 0] = s
        _check(cache, want)


@pytest.mark.parametrize("d,block", [(64, 64), (64, 128), (128, 64), (128, 128)])
def test_reading_windows(d, block):
    B, H, blocks = 5, 2, 4
    cache, want = asa.alloc_kv_cache(B, H, blocks, d, block), ref.Cache(B, H, blocks, block, d)
    _write(cache, want, _rows(1, B, H, 3 * block + 5, d, True), block, None, None)
    for L, start, count, packed in ((1, [0, 1, block, 3 * block + 4, 4 * block], None, False),
                                    (block + 9, [0, 5, block - 1, -3, 3 * block + 20], [block + 9, 0, 7, 1000, block], True),
                                    (4 * block, None, [0, 1, -2, block, 4 * block], False)):
        rows = [torch.full((B, L, H, d), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2) if packed else
                torch.full((B, H, L, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        p = asa.Params(B=B, H=H, L=L, d=d, block=block, k_stride=rows[0].stride()[:3], v_stride=rows[1].stride()[:3])
        asa.asa_cache_read(p, cache, *rows, start=None if start is None else _i32(start), count=None if count is None else _i32(count))
        for name, got in zip("kv", rows):
            expect = np.full((B, H, L, d), 7.0)
            for b in range(B):
                for r in range(min(max(count[b], 0), L) if count else L):
                    pos = r + (start[b] if start else 0)
                    if 0 <= pos < blocks * block:
                        expect[b, :, r] = want.values(name)[b, :, pos]
            assert np.array_equal(_np(got), expect), (name, L)
