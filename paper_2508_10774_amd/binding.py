"""ctypes binding of libasa.so: same entry-point names as ``include/asa.h``.

Argument marshalling only.  Tensors are torch CUDA(ROCm) tensors used for device memory
and streams; every step of the method runs in the HIP kernels of the library.  There is no
CPU or PyTorch fallback: if the library is missing or a call fails, an exception is raised.
"""

from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libasa.so")
_lib = None


class AsaError(RuntimeError):
    pass


class asa_params(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32), ("d", ctypes.c_int32),
        ("block", ctypes.c_int32), ("k_samples", ctypes.c_int32),
        ("sample_offsets", ctypes.POINTER(ctypes.c_int32)),
        ("tau", ctypes.c_float), ("r_min", ctypes.c_float), ("r_max", ctypes.c_float),
        ("n_prefix_dense", ctypes.c_int32), ("scale", ctypes.c_float),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3),
    ]


class asa_qk_norm(ctypes.Structure):
    _fields_ = [
        ("H_kv", ctypes.c_int32), ("kind", ctypes.c_int32), ("eps", ctypes.c_float), ("rot_dim", ctypes.c_int32),
        ("pairing", ctypes.c_int32), ("table_rows", ctypes.c_int32), ("first_row", ctypes.c_int32),
        ("start", ctypes.c_void_p), ("cos_table", ctypes.c_void_p), ("sin_table", ctypes.c_void_p),
        ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
        ("q_bias", ctypes.c_void_p), ("k_bias", ctypes.c_void_p),
        ("q_out_stride", ctypes.c_int64 * 3), ("k_out_stride", ctypes.c_int64 * 3),
        ("dq_stride", ctypes.c_int64 * 3), ("dk_stride", ctypes.c_int64 * 3),
    ]


class asa_kv_cache(ctypes.Structure):
    _fields_ = [
        ("H_kv", ctypes.c_int32), ("max_blocks", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
    ]


# The same fields in one call (native sizes and alignment): setting them one by one takes 4 us, as long as a launch.
_PACKED = struct.Struct("@6iP3fif12q")
assert _PACKED.size == ctypes.sizeof(asa_params)
_PACKED_NORM, _PACKED_CACHE = struct.Struct("@2if4i7P12q"), struct.Struct("@2i4P")
assert _PACKED_NORM.size == ctypes.sizeof(asa_qk_norm) and _PACKED_CACHE.size == ctypes.sizeof(asa_kv_cache)

EXPORTS = ["asa_version", "asa_error_string", "asa_last_hip_error", "asa_mask_workspace_bytes",
           "asa_fwd_workspace_bytes", "asa_bwd_workspace_bytes", "asa_build_mask",
           "asa_mask_from_scores", "asa_csr_from_mask", "asa_attn_fwd", "asa_attn_bwd",
           "asa_attn_bwd_noalloc", "asa_set_kernel_timing", "asa_global_token_count", "asa_global_tokens",
           "asa_fwd_g_workspace_bytes", "asa_attn_fwd_g", "asa_bwd_g_workspace_bytes",
           "asa_attn_bwd_g", "asa_mask_seeded_workspace_bytes", "asa_build_mask_seeded",
           "asa_sample_offsets", "asa_gilbert_order", "asa_reorder_tokens",
           "asa_qk_norm_rope", "asa_qk_norm_rope_bwd_workspace_bytes", "asa_qk_norm_rope_bwd",
           "asa_cache_write", "asa_cache_read", "asa_attn_cache_workspace_bytes", "asa_attn_cache",
           "asa_mfma_rate_probe", "asa_test_force_fwd_kernel", "asa_add_rate_probe"]


def load():
    """Load libasa.so (built by ``python -m paper_2508_10774_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise AsaError(f"{LIB_PATH} not found: build it with `python -m paper_2508_10774_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, pp = ctypes.c_void_p, ctypes.POINTER(asa_params)
    L.asa_version.restype = ctypes.c_int
    L.asa_error_string.restype = ctypes.c_char_p
    L.asa_error_string.argtypes = [ctypes.c_int]
    L.asa_last_hip_error.restype = ctypes.c_char_p
    for n in ("asa_mask_workspace_bytes", "asa_fwd_workspace_bytes", "asa_bwd_workspace_bytes",
              "asa_mask_seeded_workspace_bytes"):
        getattr(L, n).restype = ctypes.c_size_t
        getattr(L, n).argtypes = [pp]
    L.asa_build_mask.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.asa_build_mask_seeded.argtypes = [pp, ctypes.c_uint64] + [vp] * 9 + [ctypes.c_size_t, vp]
    L.asa_sample_offsets.argtypes = [pp, ctypes.c_uint64, vp, vp]
    L.asa_mask_from_scores.argtypes = [pp, vp, vp, vp]
    L.asa_csr_from_mask.argtypes = [pp, vp, vp, vp, vp, vp, vp]
    L.asa_attn_fwd.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.asa_attn_bwd.argtypes = [pp] + [vp] * 15 + [ctypes.c_size_t, vp]
    L.asa_attn_bwd_noalloc.argtypes = [pp] + [vp] * 15
    L.asa_attn_bwd_noalloc.restype = ctypes.c_int
    L.asa_set_kernel_timing.argtypes = [vp, vp]
    L.asa_add_rate_probe.argtypes = [ctypes.c_int32] * 4 + [vp, ctypes.POINTER(ctypes.c_double), vp]
    L.asa_add_rate_probe.restype = ctypes.c_int
    L.asa_test_force_fwd_kernel.argtypes = [ctypes.c_int]
    L.asa_test_force_fwd_kernel.restype = ctypes.c_int
    for n in ("asa_global_token_count", "asa_fwd_g_workspace_bytes", "asa_bwd_g_workspace_bytes"):
        getattr(L, n).restype = ctypes.c_size_t
        getattr(L, n).argtypes = [pp, ctypes.c_int]
    L.asa_global_tokens.argtypes = [pp, ctypes.c_int, vp, vp, vp, vp, vp]
    L.asa_attn_fwd_g.argtypes = [pp, ctypes.c_int] + [vp] * 11 + [ctypes.c_size_t, vp]
    L.asa_attn_bwd_g.argtypes = [pp, ctypes.c_int] + [vp] * 17 + [ctypes.c_size_t, vp]
    L.asa_mfma_rate_probe.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp,
                                      ctypes.POINTER(ctypes.c_double), vp]
    L.asa_mfma_rate_probe.restype = ctypes.c_int
    L.asa_gilbert_order.argtypes = [ctypes.c_int32] * 4 + [vp, vp]
    L.asa_reorder_tokens.argtypes = [pp, ctypes.c_int32, vp, vp, vp, vp, vp, vp]
    pn, pc = ctypes.POINTER(asa_qk_norm), ctypes.POINTER(asa_kv_cache)
    L.asa_qk_norm_rope.argtypes = [pp, pn] + [vp] * 5
    L.asa_qk_norm_rope_bwd.argtypes = [pp, pn] + [vp] * 11 + [ctypes.c_size_t, vp]
    L.asa_qk_norm_rope_bwd_workspace_bytes.argtypes = [pp, pn]
    L.asa_cache_write.argtypes = L.asa_cache_read.argtypes = [pp, pc] + [vp] * 5
    L.asa_attn_cache.argtypes = [pp, pc] + [vp] * 7 + [ctypes.c_size_t, vp]
    L.asa_attn_cache_workspace_bytes.argtypes = [pp, pc]
    for n in ("asa_qk_norm_rope_bwd_workspace_bytes", "asa_attn_cache_workspace_bytes"):
        getattr(L, n).restype = ctypes.c_size_t
    for n in ("asa_qk_norm_rope", "asa_qk_norm_rope_bwd", "asa_cache_write", "asa_cache_read", "asa_attn_cache"):
        getattr(L, n).restype = ctypes.c_int
    for n in ("asa_gilbert_order", "asa_reorder_tokens", "asa_build_mask", "asa_mask_from_scores", "asa_csr_from_mask", "asa_attn_fwd",
              "asa_attn_bwd", "asa_set_kernel_timing", "asa_global_tokens", "asa_attn_fwd_g",
              "asa_attn_bwd_g", "asa_build_mask_seeded", "asa_sample_offsets"):
        getattr(L, n).restype = ctypes.c_int
    _lib = L
    return L


@dataclass
class Params:
    """Python mirror of ``asa_params``; ``c()`` builds the C struct (keeps offsets alive)."""
    B: int
    H: int
    L: int
    d: int
    block: int
    k_samples: int = 16
    sample_offsets: Optional[Sequence[int]] = None
    tau: float = 0.9
    r_min: float = 0.0
    r_max: float = 1.0
    n_prefix_dense: int = 0
    scale: float = 0.0
    q_stride: Sequence[int] = (0, 0, 0)
    k_stride: Sequence[int] = (0, 0, 0)
    v_stride: Sequence[int] = (0, 0, 0)
    o_stride: Sequence[int] = (0, 0, 0)

    @property
    def Nb(self) -> int:
        return (self.L + self.block - 1) // self.block

    def c(self) -> asa_params:
        if self.sample_offsets is None:
            try:
                (q0, q1, q2), (k0, k1, k2), (v0, v1, v2), (o0, o1, o2) = self.q_stride, self.k_stride, self.v_stride, self.o_stride
                return asa_params.from_buffer_copy(_PACKED.pack(
                    self.B, self.H, self.L, self.d, self.block, self.k_samples, 0, self.tau, self.r_min, self.r_max,
                    self.n_prefix_dense, self.scale, q0, q1, q2, k0, k1, k2, v0, v1, v2, o0, o1, o2))
            except (struct.error, TypeError, ValueError, OverflowError):
                pass            # values that want converting, or that ctypes refuses: one by one
        p = asa_params()
        p.B, p.H, p.L, p.d, p.block, p.k_samples = self.B, self.H, self.L, self.d, self.block, self.k_samples
        if self.sample_offsets is not None:
            arr = (ctypes.c_int32 * len(self.sample_offsets))(*[int(x) for x in self.sample_offsets])
            p._keep = arr
            p.sample_offsets = ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32))
        p.tau, p.r_min, p.r_max = self.tau, self.r_min, self.r_max
        p.n_prefix_dense, p.scale = self.n_prefix_dense, self.scale
        for name in ("q_stride", "k_stride", "v_stride", "o_stride"):
            setattr(p, name, (ctypes.c_int64 * 3)(*[int(x) for x in getattr(self, name)]))
        return p


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise AsaError("libasa takes device tensors")
    return t.data_ptr()


# (the stream's handle without a Stream object around it, where this torch has that)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _check(rc: int, what: str):
    if rc != 0:
        L = load()
        msg = L.asa_error_string(rc).decode()
        if rc == -4:
            msg += ": " + L.asa_last_hip_error().decode()
        raise AsaError(f"{what} failed ({rc}): {msg}")


def asa_version() -> int:
    return load().asa_version()


def asa_mask_workspace_bytes(p: Params) -> int:
    return load().asa_mask_workspace_bytes(ctypes.byref(p.c()))


def asa_fwd_workspace_bytes(p: Params) -> int:
    return load().asa_fwd_workspace_bytes(ctypes.byref(p.c()))


def asa_bwd_workspace_bytes(p: Params) -> int:
    return load().asa_bwd_workspace_bytes(ctypes.byref(p.c()))


def asa_build_mask(p: Params, q, k, mask, row_ptr, col_idx, col_ptr=None, row_idx=None,
                   p_imp=None, workspace=None, stream=None):
    ws_bytes = workspace.nbytes if workspace is not None else 0
    rc = load().asa_build_mask(ctypes.byref(p.c()), _ptr(q), _ptr(k), _ptr(mask), _ptr(row_ptr),
                               _ptr(col_idx), _ptr(col_ptr), _ptr(row_idx), _ptr(p_imp),
                               _ptr(workspace), ws_bytes, _stream(stream))
    _check(rc, "asa_build_mask")


def asa_mask_from_scores(p: Params, scores, mask, stream=None):
    _check(load().asa_mask_from_scores(ctypes.byref(p.c()), _ptr(scores), _ptr(mask),
                                       _stream(stream)), "asa_mask_from_scores")


def asa_csr_from_mask(p: Params, mask, row_ptr, col_idx, col_ptr=None, row_idx=None, stream=None):
    _check(load().asa_csr_from_mask(ctypes.byref(p.c()), _ptr(mask), _ptr(row_ptr), _ptr(col_idx),
                                    _ptr(col_ptr), _ptr(row_idx), _stream(stream)),
           "asa_csr_from_mask")


def asa_attn_fwd(p: Params, q, k, v, row_ptr, col_idx, o, lse, workspace, o_lo=None, stream=None):
    ws_bytes = workspace.nbytes if workspace is not None else 0
    _check(load().asa_attn_fwd(ctypes.byref(p.c()), _ptr(q), _ptr(k), _ptr(v), _ptr(row_ptr),
                               _ptr(col_idx), _ptr(o), _ptr(o_lo), _ptr(lse), _ptr(workspace),
                               ws_bytes, _stream(stream)), "asa_attn_fwd")


def asa_attn_bwd(p: Params, q, k, v, o, d_o, lse, row_ptr, col_idx, col_ptr, row_idx, dq, dk, dv,
                 workspace, o_lo=None, stream=None):
    ws_bytes = workspace.nbytes if workspace is not None else 0
    _check(load().asa_attn_bwd(ctypes.byref(p.c()), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(o_lo),
                               _ptr(d_o), _ptr(lse), _ptr(row_ptr), _ptr(col_idx), _ptr(col_ptr),
                               _ptr(row_idx), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
                               ws_bytes, _stream(stream)), "asa_attn_bwd")


def asa_add_rate_probe(atomic: bool, workgroups: int, tiles_per_workgroup: int, n_qblocks: int, buf,
                       stream=None) -> float:
    """asa_bench.h: launches the calibration kernel; returns the payload bytes of the launch."""
    b = ctypes.c_double()
    _check(load().asa_add_rate_probe(int(bool(atomic)), workgroups, tiles_per_workgroup, n_qblocks,
                                     _ptr(buf), ctypes.byref(b), _stream(stream)), "asa_add_rate_probe")
    return b.value


def asa_test_force_fwd_kernel(which: int):
    """asa_bench.h: 0 = the library's choice, 1 = lock-step kernel, 2 = ping-pong kernel, 4 = wide kernel."""
    _check(load().asa_test_force_fwd_kernel(int(which)), "asa_test_force_fwd_kernel")


NOALLOC_SCRATCH_BYTES = 8 << 20   # ASA_NOALLOC_SCRATCH_BYTES of asa.h


def asa_attn_bwd_noalloc(p: Params, q, k, v, o, d_o, lse, row_ptr, col_idx, col_ptr, row_idx, dq,
                         dk, dv, o_lo=None, stream=None):
    _check(load().asa_attn_bwd_noalloc(ctypes.byref(p.c()), _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                       _ptr(o_lo), _ptr(d_o), _ptr(lse), _ptr(row_ptr),
                                       _ptr(col_idx), _ptr(col_ptr), _ptr(row_idx), _ptr(dq),
                                       _ptr(dk), _ptr(dv), _stream(stream)), "asa_attn_bwd_noalloc")


def asa_mask_seeded_workspace_bytes(p: Params) -> int:
    return int(load().asa_mask_seeded_workspace_bytes(ctypes.byref(p.c())))


def asa_build_mask_seeded(p: Params, seed: int, q, k, mask, row_ptr, col_idx, col_ptr, row_idx,
                          p_imp, workspace, stream=None):
    ws_bytes = workspace.nbytes if workspace is not None else 0
    _check(load().asa_build_mask_seeded(ctypes.byref(p.c()), seed, _ptr(q), _ptr(k), _ptr(mask),
                                        _ptr(row_ptr), _ptr(col_idx), _ptr(col_ptr), _ptr(row_idx),
                                        _ptr(p_imp), _ptr(workspace), ws_bytes, _stream(stream)),
           "asa_build_mask_seeded")


def asa_sample_offsets(p: Params, seed: int, table, stream=None):
    _check(load().asa_sample_offsets(ctypes.byref(p.c()), seed, _ptr(table), _stream(stream)),
           "asa_sample_offsets")


def asa_global_token_count(p: Params, n: int) -> int:
    return int(load().asa_global_token_count(ctypes.byref(p.c()), n))


def asa_global_tokens(p: Params, n: int, k, v, kg, vg, stream=None):
    _check(load().asa_global_tokens(ctypes.byref(p.c()), n, _ptr(k), _ptr(v), _ptr(kg), _ptr(vg),
                                    _stream(stream)), "asa_global_tokens")


def asa_fwd_g_workspace_bytes(p: Params, n: int) -> int:
    return int(load().asa_fwd_g_workspace_bytes(ctypes.byref(p.c()), n))


def asa_attn_fwd_g(p: Params, n: int, q, k, v, kg, vg, row_ptr, col_idx, o, lse, workspace,
                   o_lo=None, stream=None):
    ws_bytes = workspace.nbytes if workspace is not None else 0
    _check(load().asa_attn_fwd_g(ctypes.byref(p.c()), n, _ptr(q), _ptr(k), _ptr(v), _ptr(kg),
                                 _ptr(vg), _ptr(row_ptr), _ptr(col_idx), _ptr(o), _ptr(o_lo),
                                 _ptr(lse), _ptr(workspace), ws_bytes, _stream(stream)),
           "asa_attn_fwd_g")


def asa_bwd_g_workspace_bytes(p: Params, n: int) -> int:
    return int(load().asa_bwd_g_workspace_bytes(ctypes.byref(p.c()), n))


def asa_attn_bwd_g(p: Params, n: int, q, k, v, kg, vg, o, d_o, lse, row_ptr, col_idx, col_ptr,
                   row_idx, dq, dk, dv, workspace, o_lo=None, stream=None):
    ws_bytes = workspace.nbytes if workspace is not None else 0
    _check(load().asa_attn_bwd_g(ctypes.byref(p.c()), n, _ptr(q), _ptr(k), _ptr(v), _ptr(kg),
                                 _ptr(vg), _ptr(o), _ptr(o_lo), _ptr(d_o), _ptr(lse), _ptr(row_ptr),
                                 _ptr(col_idx), _ptr(col_ptr), _ptr(row_idx), _ptr(dq), _ptr(dk),
                                 _ptr(dv), _ptr(workspace), ws_bytes, _stream(stream)),
           "asa_attn_bwd_g")


def asa_gilbert_order(T: int, Y: int, X: int, n_prefix: int = 0):
    """(order, inverse) as int32 CPU tensors of n_prefix + T*Y*X entries (host function)."""
    n = max(0, n_prefix) + max(0, T) * max(0, Y) * max(0, X)
    order = torch.empty(n, dtype=torch.int32)
    inverse = torch.empty(n, dtype=torch.int32)
    _check(load().asa_gilbert_order(T, Y, X, n_prefix, ctypes.c_void_p(order.data_ptr()),
                                    ctypes.c_void_p(inverse.data_ptr())), "asa_gilbert_order")
    return order, inverse


def asa_reorder_tokens(p: Params, src, dst, index, src_stride=None, dst_stride=None, stream=None):
    """dst[t][b, h, i, :] = src[t][b, h, index[i], :] for lists of up to three tensors."""
    n = len(src)
    if len(dst) != n:
        raise AsaError("asa_reorder_tokens: src and dst differ in length")
    srcs = (ctypes.c_void_p * n)(*[t.data_ptr() for t in src])
    dsts = (ctypes.c_void_p * n)(*[t.data_ptr() for t in dst])
    ss = (ctypes.c_int64 * 3)(*src_stride) if src_stride is not None else None
    ds = (ctypes.c_int64 * 3)(*dst_stride) if dst_stride is not None else None
    _check(load().asa_reorder_tokens(ctypes.byref(p.c()), n, srcs, dsts, ss, ds, _ptr(index),
                                     _stream(stream)), "asa_reorder_tokens")


# ---------------------------------------------------------------------------
# norm and rotation of queries and keys; keys and values in 8 bits
# ---------------------------------------------------------------------------

# (the current device without the checks of torch.cuda around it: a device tensor is at hand when it is asked for)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _device(stream, first: Optional[torch.Tensor]) -> int:
    """The device that the call's tensors have to be on: the current one, also for a stream of the caller's."""
    if first is None or not first.is_cuda:
        raise AsaError("libasa takes device tensors")
    dev = _current_device()
    if stream is not None and stream.device_index != dev:
        raise AsaError("the stream is not one of the current device")
    return dev


def _stream_on(stream, dev: int) -> int:
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _flat(t: Optional[torch.Tensor], what: str, dtype, n: int, dev: int) -> int:
    """Pointer of a contiguous tensor of (at least) n elements; 0 for None."""
    if t is None:
        return 0
    if t.dtype is dtype and t.get_device() == dev and t.numel() >= n and t.is_contiguous():
        return t.data_ptr()
    raise AsaError(f"{what}: {n} contiguous elements of {dtype} on device {dev} expected, got {tuple(t.shape)} of {t.dtype} "
                   f"on {t.device}")


def _packed(struct_type, layout, values):
    try:
        return struct_type.from_buffer_copy(layout.pack(*values))
    except (struct.error, TypeError, OverflowError) as e:
        raise AsaError(f"{struct_type.__name__}: {e}") from None


def _rows(t: Optional[torch.Tensor], what: str, shape, stride, dev: int) -> int:
    """Pointer of a bf16 tensor [B, heads, L, d] that has the strides that the call gives for it; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not torch.bfloat16 or t.get_device() != dev or t.shape != shape:
        raise AsaError(f"{what}: bf16 {shape} on device {dev} expected, got {tuple(t.shape)} of {t.dtype} on {t.device}")
    s0, s1, s2 = stride
    if not (s0 or s1 or s2):
        s2 = shape[3]
        s1 = shape[2] * s2
        s0 = shape[1] * s1
    got = t.stride()
    if got != (s0, s1, s2, 1) and any(n > 1 and a != b for n, a, b in zip(shape, got, (s0, s1, s2, 1))):
        raise AsaError(f"{what}: strides {(s0, s1, s2, 1)} expected, got {got}")
    return t.data_ptr()


def _own_strides(t: Optional[torch.Tensor], what: str, shape):
    """Strides of batch, head and token that a tensor [B, heads, L, d] has itself (d where there is one: it says nothing); zeros for None."""
    if t is None or t.dim() != 4:
        return 0, 0, 0
    d, got = shape[3], t.stride()
    if got[3] != 1 or any(n > 1 and s < d for n, s in zip(shape[:3], got)):
        raise AsaError(f"{what}: strides of rows that lie apart expected, got {got}")
    return tuple(s if n > 1 else d for n, s in zip(shape[:3], got))


_KINDS = {"rms": 0, "layer": 1}
_PAIRINGS = {"adjacent": 0, "halves": 1}


@dataclass
class QkNorm:
    """``asa_qk_norm``: the norm of each head's rows, its parameters, the angles of the positions.

    kind "rms" | "layer"; weights and biases [d] fp32 (None: ones, zeros); cos, sin [table_rows, rot_dim / 2] fp32;
    pairing "adjacent" | "halves"; start [B] int32, added to first_row for each sequence."""
    H_kv: int = 0
    kind: str = "rms"
    eps: float = 1e-6
    q_weight: Optional[torch.Tensor] = None
    k_weight: Optional[torch.Tensor] = None
    q_bias: Optional[torch.Tensor] = None
    k_bias: Optional[torch.Tensor] = None
    rot_dim: int = 0
    pairing: str = "adjacent"
    cos: Optional[torch.Tensor] = None
    sin: Optional[torch.Tensor] = None
    first_row: int = 0
    start: Optional[torch.Tensor] = None
    q_out_stride: Sequence[int] = (0, 0, 0)
    k_out_stride: Sequence[int] = (0, 0, 0)

    def c(self, p: Params, dev: int, dq_stride=(0, 0, 0), dk_stride=(0, 0, 0)) -> asa_qk_norm:
        if self.kind not in _KINDS or self.pairing not in _PAIRINGS:
            raise AsaError(f"kind {self.kind!r}: one of {list(_KINDS)}; pairing {self.pairing!r}: one of {list(_PAIRINGS)}")
        f32, d, rot = torch.float32, p.d, self.rot_dim
        rows = cos = sin = 0
        if rot and self.cos is not None and self.sin is not None:
            shape = self.cos.shape
            if len(shape) != 2 or shape[1] * 2 != rot or self.sin.shape != shape:
                raise AsaError(f"cos, sin: [rows, {rot // 2}] expected, got {tuple(shape)} and {tuple(self.sin.shape)}")
            rows = shape[0]
            cos, sin = _flat(self.cos, "cos", f32, 0, dev), _flat(self.sin, "sin", f32, 0, dev)
        start, qw, kw, qb, kb = self.start, self.q_weight, self.k_weight, self.q_bias, self.k_bias
        q_out, k_out = self.q_out_stride, self.k_out_stride
        return _packed(asa_qk_norm, _PACKED_NORM, (
            self.H_kv, _KINDS[self.kind], self.eps, rot, _PAIRINGS[self.pairing], rows, self.first_row,
            0 if start is None else _flat(start, "start", torch.int32, p.B, dev), cos, sin,
            0 if qw is None else _flat(qw, "q_weight", f32, d, dev), 0 if kw is None else _flat(kw, "k_weight", f32, d, dev),
            0 if qb is None else _flat(qb, "q_bias", f32, d, dev), 0 if kb is None else _flat(kb, "k_bias", f32, d, dev),
            q_out[0], q_out[1], q_out[2], k_out[0], k_out[1], k_out[2], *dq_stride, *dk_stride))


def asa_qk_norm_rope(p: Params, n: QkNorm, q, k, q_out, k_out, stream=None):
    """q [B, H, L, d], k [B, H_kv, L, d] -> q_out, k_out: norm for each head, then rotation (k = k_out = None: q alone)."""
    dev = _device(stream, q)
    qs, ks = (p.B, p.H, p.L, p.d), (p.B, n.H_kv or p.H, p.L, p.d)
    _check(load().asa_qk_norm_rope(ctypes.byref(p.c()), ctypes.byref(n.c(p, dev)), _rows(q, "q", qs, p.q_stride, dev),
                                   _rows(k, "k", ks, p.k_stride, dev), _rows(q_out, "q_out", qs, n.q_out_stride, dev),
                                   _rows(k_out, "k_out", ks, n.k_out_stride, dev), _stream_on(stream, dev)), "asa_qk_norm_rope")


def asa_qk_norm_rope_bwd_workspace_bytes(p: Params, n: QkNorm) -> int:
    """Depends on p's sizes and on n.H_kv."""
    s, c = asa_params(B=p.B, H=p.H, L=p.L, d=p.d), asa_qk_norm(H_kv=n.H_kv)
    return int(load().asa_qk_norm_rope_bwd_workspace_bytes(ctypes.byref(s), ctypes.byref(c)))


def asa_qk_norm_rope_bwd(p: Params, n: QkNorm, q, k, dq_out, dk_out, dq, dk, dq_weight, dk_weight, dq_bias, dk_bias,
                         workspace, stream=None):
    """The gradients of q and k, and of the parameters: dq and dk in the strides that they have themselves."""
    dev = _device(stream, q)
    qs, ks = (p.B, p.H, p.L, p.d), (p.B, n.H_kv or p.H, p.L, p.d)
    f32, d = torch.float32, p.d
    dqs, dks = _own_strides(dq, "dq", qs), _own_strides(dk, "dk", ks)
    _check(load().asa_qk_norm_rope_bwd(
        ctypes.byref(p.c()), ctypes.byref(n.c(p, dev, dqs, dks)), _rows(q, "q", qs, p.q_stride, dev), _rows(k, "k", ks, p.k_stride, dev),
        _rows(dq_out, "dq_out", qs, n.q_out_stride, dev), _rows(dk_out, "dk_out", ks, n.k_out_stride, dev),
        _rows(dq, "dq", qs, dqs, dev), _rows(dk, "dk", ks, dks, dev),
        _flat(dq_weight, "dq_weight", f32, d, dev), _flat(dk_weight, "dk_weight", f32, d, dev),
        _flat(dq_bias, "dq_bias", f32, d, dev), _flat(dk_bias, "dk_bias", f32, d, dev),
        _flat(workspace, "workspace", torch.uint8, 0, dev), workspace.nbytes if workspace is not None else 0,
        _stream_on(stream, dev)), "asa_qk_norm_rope_bwd")


@dataclass
class KvCache:
    """``asa_kv_cache``: the tensors of ``alloc_kv_cache`` (k [B, H_kv, max_blocks, block/32, d/16, 32, 16] and
    v [B, H_kv, max_blocks, block/32, d/32, 2, 32, 16] uint8, the scales [B, H_kv, max_blocks] fp32)."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    @property
    def H_kv(self) -> int:
        return self.k_scale.shape[1]

    @property
    def max_blocks(self) -> int:
        return self.k_scale.shape[2]

    def c(self, p: Params, dev: int) -> asa_kv_cache:
        shape = self.k_scale.shape
        B, H, blocks = shape
        if B != p.B or self.v_scale.shape != shape:
            raise AsaError(f"cache of {tuple(shape)} and {tuple(self.v_scale.shape)} blocks for {p.B} sequences")
        codes = B * H * blocks * p.block * p.d
        if self.k.numel() != codes or self.v.numel() != codes:
            raise AsaError(f"cache: {codes} codes expected, got {self.k.numel()} and {self.v.numel()}")
        u8, f32 = torch.uint8, torch.float32
        return _packed(asa_kv_cache, _PACKED_CACHE, (
            H, blocks, _flat(self.k, "cache.k", u8, 0, dev), _flat(self.v, "cache.v", u8, 0, dev),
            _flat(self.k_scale, "cache.k_scale", f32, 0, dev), _flat(self.v_scale, "cache.v_scale", f32, 0, dev)))


def _cache_call(fn, p: Params, c: KvCache, k, v, start, count, stream):
    dev = _device(stream, c.k)
    B, i32 = p.B, torch.int32
    shape = (B, c.H_kv, p.L, p.d)
    _check(getattr(load(), fn)(ctypes.byref(p.c()), ctypes.byref(c.c(p, dev)), _rows(k, "k", shape, p.k_stride, dev),
                               _rows(v, "v", shape, p.v_stride, dev), _flat(start, "start", i32, B, dev),
                               _flat(count, "count", i32, B, dev), _stream_on(stream, dev)), fn)


def asa_cache_write(p: Params, c: KvCache, k, v, start=None, count=None, stream=None):
    """New tokens k, v [B, H_kv, L, d] to positions start[b] .. start[b] + count[b] - 1 (None: 0, L) of each sequence."""
    _cache_call("asa_cache_write", p, c, k, v, start, count, stream)


def asa_cache_read(p: Params, c: KvCache, k, v, start=None, count=None, stream=None):
    """Those positions back into rows 0 .. count[b] - 1 of k, v [B, H_kv, L, d] bf16."""
    _cache_call("asa_cache_read", p, c, k, v, start, count, stream)


def asa_attn_cache_workspace_bytes(p: Params, c: KvCache) -> int:
    """Depends on p's sizes and strides and on the cache's heads and blocks (0: no workspace needed)."""
    s = asa_kv_cache(H_kv=c.H_kv, max_blocks=c.max_blocks)
    return int(load().asa_attn_cache_workspace_bytes(ctypes.byref(p.c()), ctypes.byref(s)))


def asa_attn_cache(p: Params, c: KvCache, length, q, row_ptr, col_idx, o, lse, workspace, stream=None):
    """q [B, H, L, d] attends to tokens [0, length[b]) of the cache, in the blocks of the lists if there are any."""
    dev = _device(stream, q)
    shape, i32 = (p.B, p.H, p.L, p.d), torch.int32
    ptr = idx = 0
    if row_ptr is not None or col_idx is not None:
        lists, rows = p.B * c.H_kv, p.Nb
        ptr = _flat(row_ptr, "row_ptr", i32, lists * (rows + 1), dev)
        idx = _flat(col_idx, "col_idx", i32, lists * rows * c.max_blocks, dev)
    _check(load().asa_attn_cache(
        ctypes.byref(p.c()), ctypes.byref(c.c(p, dev)), _flat(length, "length", i32, p.B, dev), _rows(q, "q", shape, p.q_stride, dev),
        ptr, idx, _rows(o, "o", shape, p.o_stride, dev), _flat(lse, "lse", torch.float32, p.B * p.H * p.L, dev),
        _flat(workspace, "workspace", torch.uint8, 0, dev), workspace.nbytes if workspace is not None else 0,
        _stream_on(stream, dev)), "asa_attn_cache")


def asa_mfma_rate_probe(workgroups: int, iters: int, sink, idle_sleep: int = 0, vector_stream: bool = False,
                        stream=None) -> float:
    """Launch the MFMA-only calibration kernel; returns the FLOP of the launch."""
    flop = ctypes.c_double(0.0)
    _check(load().asa_mfma_rate_probe(workgroups, iters, idle_sleep, int(vector_stream), _ptr(sink),
                                      ctypes.byref(flop), _stream(stream)), "asa_mfma_rate_probe")
    return flop.value


def asa_set_kernel_timing(start: Optional[torch.cuda.Event], stop: Optional[torch.cuda.Event]):
    """Arm the one-shot hook with two torch events (they must have been recorded once, which
    is what creates their HIP handles)."""
    a = ctypes.c_void_p(start.cuda_event) if start is not None else None
    b = ctypes.c_void_p(stop.cuda_event) if stop is not None else None
    _check(load().asa_set_kernel_timing(a, b), "asa_set_kernel_timing")


# ---------------------------------------------------------------------------
# device-memory helpers (allocation only)
# ---------------------------------------------------------------------------

def alloc_index_lists(p: Params, device="cuda", with_csc: bool = True):
    """Empty mask / CSR / CSC buffers of the sizes ``asa.h`` documents."""
    S, Nb = p.B * p.H, p.Nb
    out = {
        "mask": torch.empty((S, Nb, Nb), dtype=torch.uint8, device=device),
        "row_ptr": torch.empty((S, Nb + 1), dtype=torch.int32, device=device),
        "col_idx": torch.empty((S, Nb * Nb), dtype=torch.int32, device=device),
    }
    if with_csc:
        out["col_ptr"] = torch.empty((S, Nb + 1), dtype=torch.int32, device=device)
        out["row_idx"] = torch.empty((S, Nb * Nb), dtype=torch.int32, device=device)
    return out


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty((max(int(nbytes), 256),), dtype=torch.uint8, device=device)


def alloc_kv_cache(B: int, H_kv: int, max_blocks: int, d: int, block: int, device="cuda") -> KvCache:
    """An empty cache: room for max_blocks * block tokens of each sequence, all zeros at the scale that the writer gives zeros (a
    larger one would stay where a sequence begins behind tokens that were never written, and cost what follows its precision)."""
    lead = (B, H_kv, max_blocks)
    k = torch.zeros(*lead, block // 32, d // 16, 32, 16, dtype=torch.uint8, device=device)
    v = torch.zeros(*lead, block // 32, d // 32, 2, 32, 16, dtype=torch.uint8, device=device)
    k_scale, v_scale = (torch.full(lead, 2.0 ** -100, dtype=torch.float32, device=device) for _ in range(2))
    return KvCache(k, v, k_scale, v_scale)
