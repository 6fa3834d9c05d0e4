"""What the binding of the norm, cache and cached-attention calls raises where the tensor is missing that the device is taken from (no GPU)."""

import pytest

from paper_2508_10774_amd import binding

P = binding.Params(B=1, H=2, L=4, d=64, block=64)


def test_missing_tensors_raise_the_librarys_error():
    cache = binding.KvCache(None, None, None, None)
    whole = binding.alloc_kv_cache(1, 2, 1, 64, 64, device="cpu")
    calls = [lambda: binding.asa_qk_norm_rope(P, binding.QkNorm(), None, None, None, None),
             lambda: binding.asa_qk_norm_rope_bwd(P, binding.QkNorm(), *[None] * 11),
             lambda: binding.asa_cache_write(P, cache, None, None),
             lambda: binding.asa_cache_read(P, cache, None, None),
             lambda: binding.asa_attn_cache(P, whole, None, None, None, None, None, None, None)]
    for call in calls:
        with pytest.raises(binding.AsaError, match="device tensors"):
            call()
