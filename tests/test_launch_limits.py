"""Calls of more work than one launch holds (2^32 - 1 threads along an axis) are refused as such, before anything is launched (no
GPU needed: the pointers are never used)."""

import ctypes

import pytest
import torch

from paper_2508_10774_amd import binding

FAKE = ctypes.c_void_p(0x10000)
UNSUPPORTED, HIP = -2, -4


def _params(B, H, L, d, block):
    return ctypes.byref(binding.Params(B=B, H=H, L=L, d=d, block=block).c())


def _cache(H_kv, max_blocks):
    return ctypes.byref(binding.asa_kv_cache(H_kv=H_kv, max_blocks=max_blocks, k=0x1000, v=0x2000, k_scale=0x3000, v_scale=0x4000))


@pytest.mark.parametrize("B,H,L,d", [(1 << 16, 1, 1 << 12, 128), (1 << 13, 1, 1 << 16, 64), (1 << 22, 256, 1, 64), (1 << 20, 1, 257, 128)])
def test_norm(B, H, L, d):
    """256 threads for 16 tokens of 4 heads of 128, 32 tokens of 4 heads of 64."""
    n = binding.asa_qk_norm(H_kv=H)
    L_ = binding.load()
    assert L_.asa_qk_norm_rope(_params(B, H, L, d, 128), ctypes.byref(n), FAKE, None, FAKE, None, None) == UNSUPPORTED


def test_norm_of_queries_and_keys_together():
    """Each of them alone is a launch of 2^23 workgroups."""
    n = binding.asa_qk_norm(H_kv=1)
    assert binding.load().asa_qk_norm_rope(_params(1 << 15, 1, 1 << 12, 128, 128), ctypes.byref(n), *[FAKE] * 4, None) == UNSUPPORTED


@pytest.mark.parametrize("fn", ["asa_cache_write", "asa_cache_read"])
@pytest.mark.parametrize("B,H,blocks,d,block,sides", [(1 << 16, 256, 1, 64, 128, 1), (1 << 16, 128, 1, 128, 64, 2), (1 << 17, 256, 1, 64, 64, 1),
                                                      (1 << 12, 64, 128, 128, 128, 1)])
def test_cache(fn, B, H, blocks, d, block, sides):
    """256 threads for a block of either tensor, 128 at block 64 / d 64."""
    L = block * blocks
    c = _cache(H, blocks)
    assert getattr(binding.load(), fn)(_params(B, H, L, d, block), c, FAKE, FAKE if sides == 2 else None, None, None, None) == UNSUPPORTED


@pytest.mark.parametrize("B,H,H_kv,L", [(1 << 22, 4, 4, 1), (1 << 25, 1, 1, 64), (1 << 14, 1 << 15, 1 << 12, 64)])
def test_cached_attention(B, H, H_kv, L):
    """256 threads for a tile of up to 32 rows, 128 for one of up to 64, 256 for one of up to 128."""
    rc = binding.load().asa_attn_cache(_params(B, H, L, 64, 64), _cache(H_kv, 1), FAKE, FAKE, None, None, FAKE, FAKE, FAKE, 1 << 45, None)
    assert rc == UNSUPPORTED


@pytest.mark.skipif(torch.cuda.is_available(), reason="would launch: the calls end for want of a device")
def test_the_largest_launches_pass_the_checks():
    L = binding.load()
    n = binding.asa_qk_norm(H_kv=1)
    assert L.asa_qk_norm_rope(_params((1 << 21) - 1, 1, 256, 64, 64), ctypes.byref(n), FAKE, None, FAKE, None, None) == HIP
    c = _cache(1, 1)
    assert L.asa_cache_write(_params((1 << 24) - 1, 1, 64, 64, 128), c, FAKE, None, None, None, None) == HIP
    assert L.asa_cache_read(_params((1 << 25) - 1, 1, 64, 64, 64), c, FAKE, None, None, None, None) == HIP
    assert L.asa_attn_cache(_params((1 << 24) - 8, 1, 1, 64, 64), c, FAKE, FAKE, None, None, FAKE, FAKE, None, 0, None) == HIP
    assert L.asa_attn_cache(_params((1 << 25) - 8, 1, 64, 64, 64), c, FAKE, FAKE, None, None, FAKE, FAKE, None, 0, None) == HIP


def test_the_backwards_launch_does_not_grow():
    """(its workgroups walk: more rows than the forward takes)"""
    n = binding.asa_qk_norm(H_kv=1)
    assert binding.load().asa_qk_norm_rope_bwd_workspace_bytes(_params(1 << 16, 1, 1 << 12, 128, 128), ctypes.byref(n)) > 0
