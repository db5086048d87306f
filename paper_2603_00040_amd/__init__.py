"""Thin Python binding of the gfx950 Attn-QAT C ABI (``include/attnqat.h``).

Argument marshalling only: every step of the path runs in the HIP kernels of
``libattnqat.so``.  PyTorch supplies device memory and the current stream.
There is no CPU or PyTorch fallback: if the shared library is missing, loading
fails with an error that says how to build it.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libattnqat.so")

OK, EINVAL, ESHAPE, EDTYPE, EWORKSPACE, ELAUNCH, ESTATIC = 0, -1, -2, -3, -4, -5, -6
STATIC_SCRATCH_BYTES = 32 << 20
BF16 = 0
(WS_FWD, WS_FWD_INFER, WS_BWD, WS_FWD_INFER_MX, WS_FWD_MX, WS_BWD_MX, WS_FWD_INFER_MX_FP8PV,
 WS_FWD_INFER_MX_PAGED, WS_FWD_INFER_MX_SPARSE) = 0, 1, 2, 3, 4, 5, 6, 7, 8

_vp, _i, _sz, _ll, _f = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_int64, ctypes.c_float
_SIGNATURES = {
    "attnqat_quantize": (_i, [_vp, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "attnqat_fwd": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_fwd_infer": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_fwd_infer_bf16pv": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_fwd_infer_static": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp]),
    "attnqat_fwd_infer_packed": (_i, [_vp] * 6 + [_i] * 7 + [_vp, _vp, _vp, _sz, _vp]),
    "attnqat_bwd_packed": (_i, [_vp] * 9 + [_i] * 7 + [_vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_bwd": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i,
                         _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_bwd_ablation": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _i,
                                  _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_quantize_mx": (_i, [_vp, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "attnqat_fwd_infer_mx": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_quantize_mxfp8": (_i, [_vp, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "attnqat_fwd_infer_mx_fp8pv": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_fwd_opt": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_bwd_opt": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _i,
                             _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_debug_fwd_p_opt": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _i, _vp,
                                     _vp, _sz, _vp]),
    "attnqat_kv_cache_page_bytes": (_sz, [_i, _i]),
    "attnqat_kv_cache_write_mx": (_i, [_vp, _vp, _i, _i, _i, _i, _vp, _i, _vp, _vp]),
    "attnqat_fwd_infer_mx_paged": (_i, [_vp, _i, _i, _i, _i, _i, _i, _i, _vp, _i, _vp, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_kv_cache_page_bytes_nvfp4": (_sz, [_i, _i]),
    "attnqat_kv_cache_write": (_i, [_vp, _vp, _i, _i, _i, _i, _i, _vp, _i, _vp, _vp]),
    "attnqat_paged_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "attnqat_fwd_infer_paged": (_i, [_vp, _i, _i, _i, _i, _i, _i, _i, _vp, _i, _vp, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_debug_fwd_infer_paged": (_i, [_vp, _i, _i, _i, _i, _i, _i, _i, _vp, _i, _vp, _i, _vp, _vp, _vp, _vp, _sz, _vp, _i, _vp]),
    "attnqat_page_plan_workspace_bytes": (_sz, [_i]),
    "attnqat_page_plan": (_i, [_vp, _vp, _i, _vp, _i, _vp, _i, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_kv_cache_append": (_i, [_vp, _ll, _ll, _vp, _ll, _ll, _i, _i, _i, _i, _vp, _i, _vp, _vp]),
    "attnqat_kv_cache_read": (_i, [_vp, _i, _vp, _i, _i, _i, _i, _vp, _ll, _ll, _vp, _ll, _ll, _vp]),
    "attnqat_kv4_ragged_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i, _i]),
    "attnqat_fwd_kv4_ragged": (_i, [_vp, _ll, _ll, _vp, _i, _i, _i, _i, _i, _i, _i, _i, _f, _i, _vp, _i, _vp, _i, _vp, _vp, _ll, _ll, _vp,
                                    _vp, _sz, _vp]),
    "attnqat_rope_table": (_i, [_vp, _i, _i, _i, _vp, _vp]),
    "attnqat_rope_fwd": (_i, [_vp, _ll, _ll, _ll] * 2 + [_i] * 6 + [_vp, _ll, _vp] + [_vp, _ll, _ll, _ll] * 2 + [_vp]),
    "attnqat_rope_bwd": (_i, [_vp, _ll, _ll, _ll] * 2 + [_i] * 6 + [_vp, _ll, _vp] + [_vp, _ll, _ll, _ll] * 2 + [_vp]),
    "attnqat_kv_cache_append_rope": (_i, [_vp, _ll, _ll] * 3 + [_i] * 5 + [_vp, _vp, _vp, _i, _vp] + [_vp, _ll, _ll, _vp]),
    "attnqat_kv_summary_page_bytes": (_sz, [_i, _i]),
    "attnqat_kv_summarize": (_i, [_vp, _i, _vp, _i, _i, _i, _vp, _vp]),
    "attnqat_kv_select": (_i, [_vp, _ll, _ll, _vp] + [_i] * 7 + [_vp, _i, _vp, _i, _vp] + [_i] * 3 + [_vp, _vp]),
    "attnqat_kv4_sparse_workspace_bytes": (_sz, [_i] * 6),
    "attnqat_fwd_kv4_sparse": (_i, [_vp, _ll, _ll, _vp] + [_i] * 6 + [_f, _i, _vp, _i, _vp, _i, _vp, _vp, _i, _vp, _ll, _ll, _vp, _vp, _sz, _vp]),
    "attnqat_fwd_infer_mx_sparse": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_fwd_mx": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_bwd_mx": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i,
                            _vp, _vp, _vp, _vp, _sz, _vp]),
    "attnqat_debug_fwd_p_mx": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _i, _vp,
                                    _vp, _sz, _vp]),
    "attnqat_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i]),
    "attnqat_block_k": (_i, []),
    "attnqat_strerror": (ctypes.c_char_p, [_i]),
    "attnqat_debug_fwd_p": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _i, _vp,
                                 _vp, _sz, _vp]),
    "attnqat_debug_bwd_p": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _i, _vp, _vp, _sz, _vp]),
    "attnqat_debug_dkdv_tile_counts": (_i, [_vp, _vp]),
    "attnqat_debug_bwd_waves": (_i, [_i]),
    "attnqat_profile_enable": (_i, [_vp, _i]),
    "attnqat_profile_read": (_i, [_vp, _i, _vp, _vp]),
}
EXPORTS = tuple(_SIGNATURES)

_lib = None


class AttnQatError(RuntimeError):
    pass


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise AttnQatError(
                f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                "(hipcc --offload-arch=gfx950). There is no fallback path.")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _check(rc: int):
    if rc != OK:
        raise AttnQatError(f"attnqat error {rc}: {lib().attnqat_strerror(rc).decode()}")


def _ptr(t):
    return None if t is None else t.data_ptr()


# (the handle itself where this torch has a way to it, which is not part of its public interface: torch.cuda.current_stream() builds a
#  Stream object around it on every call, a few microseconds of a step whose kernels take twenty)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _stream_on(dev):
    return torch.cuda.current_stream(dev).cuda_stream if _raw_stream is None else _raw_stream(dev)


def _dev_bf16(t, name):
    if not (t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous() and t.dim() == 4):
        raise AttnQatError(f"{name} must be a contiguous 4-d bf16 CUDA tensor [B,H,L,d]")


def block_k() -> int:
    return lib().attnqat_block_k()


def workspace_bytes(which: int, B: int, Hq: int, Hkv: int, L: int, d: int) -> int:
    return lib().attnqat_workspace_bytes(which, B, Hq, Hkv, L, d)


def _workspace(which, B, Hq, Hkv, L, d, workspace):
    if workspace is None:
        workspace = torch.empty(max(workspace_bytes(which, B, Hq, Hkv, L, d), 1), dtype=torch.uint8, device="cuda")
    return workspace, workspace.numel()


def attnqat_quantize(x, want_codes=True, want_xf=True):
    """phi of Eq. 1 along d.  Returns (codes u8 [B,H,L,d/2], scales u8 [B,H,L,d/16], xf bf16)."""
    _dev_bf16(x, "x")
    B, H, L, d = x.shape
    codes = torch.empty((B, H, L, d // 2), dtype=torch.uint8, device=x.device) if want_codes else None
    scales = torch.empty((B, H, L, d // 16), dtype=torch.uint8, device=x.device) if want_codes else None
    xf = torch.empty_like(x) if want_xf else None
    _check(lib().attnqat_quantize(_ptr(x), B, H, L, d, BF16, _ptr(codes), _ptr(scales), _ptr(xf), _stream()))
    return codes, scales, xf


OPT_SMOOTH_K, OPT_TWO_LEVEL_P, OPT_BF16_PV = 1, 2, 4


def attnqat_fwd_infer_mx_sparse(q, k, v, causal: bool, block_mask, workspace=None, out=None):
    """Alg. 1 (MX, FP4 matrix instruction) with a block mask: uint8 CUDA tensor [B,Hq,nb,nb], nb = ceil(L/128), zero =
    the 128 x 128 block is left out.  Returns (o bf16, lse fp32)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _dev_bf16(t, n)
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    nb = (L + 127) // 128
    if not (block_mask.is_cuda and block_mask.dtype == torch.uint8 and block_mask.is_contiguous()
            and tuple(block_mask.shape) == (B, Hq, nb, nb)):
        raise AttnQatError("block_mask must be a contiguous uint8 CUDA tensor [B,Hq,ceil(L/128),ceil(L/128)]")
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
    else:
        o, lse = out
    ws, nbytes = _workspace(WS_FWD_INFER_MX_SPARSE, B, Hq, Hkv, L, d, workspace)
    _check(lib().attnqat_fwd_infer_mx_sparse(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, L, d, int(causal), BF16, _ptr(block_mask),
                                             _ptr(o), _ptr(lse), _ptr(ws), nbytes, _stream()))
    return o, lse


def kv_cache_page_bytes(Hkv: int, d: int) -> int:
    return lib().attnqat_kv_cache_page_bytes(Hkv, d)


def attnqat_kv_cache_write_mx(k, v, cache, page_ids, num_pages=None):
    """Quantize one sequence's k, v [1,Hkv,L,d] bf16 into the pages ``page_ids`` (int32 CUDA tensor) of the FP4 KV
    ``cache`` (uint8 CUDA tensor of num_pages * kv_cache_page_bytes(Hkv, d) bytes)."""
    _dev_bf16(k, "k"); _dev_bf16(v, "v")
    _, Hkv, L, d = k.shape
    if k.shape[0] != 1 or v.shape != k.shape:
        raise AttnQatError("k and v must be [1,Hkv,L,d] of one sequence")
    if not (page_ids.is_cuda and page_ids.dtype == torch.int32 and page_ids.is_contiguous() and page_ids.numel() >= (L + 127) // 128):
        raise AttnQatError("page_ids must be a contiguous int32 CUDA tensor with ceil(L/128) entries")
    if num_pages is None:
        num_pages = cache.numel() // kv_cache_page_bytes(Hkv, d)
    _check(lib().attnqat_kv_cache_write_mx(_ptr(k), _ptr(v), Hkv, L, d, BF16, _ptr(cache), int(num_pages), _ptr(page_ids), _stream()))


def attnqat_fwd_infer_mx_paged(q, cache, num_pages, page_table, kv_lens, Hkv, causal: bool, workspace=None, out=None):
    """Alg. 1 (MX, FP4 matrix instruction) over a paged FP4 KV cache.  q [B,Hq,Lq,d]: the last Lq positions of every
    sequence; page_table int32 [B,max_pages]; kv_lens int32 [B].  Returns (o bf16, lse fp32)."""
    _dev_bf16(q, "q")
    B, Hq, Lq, d = q.shape
    for t, n in ((page_table, "page_table"), (kv_lens, "kv_lens")):
        if not (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()):
            raise AttnQatError(f"{n} must be a contiguous int32 CUDA tensor")
    if page_table.dim() != 2 or page_table.shape[0] != B or kv_lens.numel() != B:
        raise AttnQatError("page_table must be [B,max_pages] and kv_lens [B]")
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=q.device)
    else:
        o, lse = out
    ws, nb = _workspace(WS_FWD_INFER_MX_PAGED, B, Hq, Hkv, Lq, d, workspace)
    _check(lib().attnqat_fwd_infer_mx_paged(_ptr(q), B, Hq, Hkv, Lq, d, int(causal), BF16, _ptr(cache), int(num_pages),
                                            _ptr(page_table), page_table.shape[1], _ptr(kv_lens),
                                            _ptr(o), _ptr(lse), _ptr(ws), nb, _stream()))
    return o, lse


def kv_cache_page_bytes_nvfp4(Hkv: int, d: int) -> int:
    return lib().attnqat_kv_cache_page_bytes_nvfp4(Hkv, d)


def attnqat_kv_cache_write(k, v, cache, page_ids, pos0: int = 0, num_pages=None):
    """Quantize positions pos0 .. pos0+n-1 of one sequence, k, v [1,Hkv,n,d] bf16, into the pages ``page_ids`` (int32 CUDA
    tensor, the sequence's page list from its first page on) of the NVFP4 KV ``cache`` (uint8 CUDA tensor)."""
    _dev_bf16(k, "k"); _dev_bf16(v, "v")
    _, Hkv, n, d = k.shape
    if k.shape[0] != 1 or v.shape != k.shape:
        raise AttnQatError("k and v must be [1,Hkv,n,d] of one sequence")
    if not (page_ids.is_cuda and page_ids.dtype == torch.int32 and page_ids.is_contiguous() and page_ids.numel() >= (pos0 + n + 127) // 128):
        raise AttnQatError("page_ids must be a contiguous int32 CUDA tensor with ceil((pos0+n)/128) entries")
    if num_pages is None:
        num_pages = cache.numel() // kv_cache_page_bytes_nvfp4(Hkv, d)
    _check(lib().attnqat_kv_cache_write(_ptr(k), _ptr(v), Hkv, n, d, BF16, int(pos0), _ptr(cache), int(num_pages), _ptr(page_ids), _stream()))


def attnqat_fwd_infer_paged(q, cache, num_pages, page_table, kv_lens, Hkv, causal: bool, workspace=None, out=None, spin_limit=None):
    """Alg. 1 over a paged NVFP4 KV cache.  q [B,Hq,Lq,d]: the last Lq positions of every sequence; page_table int32
    [B,max_pages]; kv_lens int32 [B].  Returns (o bf16, lse fp32); with spin_limit (test hook) also whether a wait of the
    decode path expired."""
    _dev_bf16(q, "q")
    B, Hq, Lq, d = q.shape
    for t, n in ((page_table, "page_table"), (kv_lens, "kv_lens")):
        if not (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()):
            raise AttnQatError(f"{n} must be a contiguous int32 CUDA tensor")
    if page_table.dim() != 2 or page_table.shape[0] != B or kv_lens.numel() != B:
        raise AttnQatError("page_table must be [B,max_pages] and kv_lens [B]")
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=q.device)
    else:
        o, lse = out
    max_pages = page_table.shape[1]
    if workspace is None:
        need = lib().attnqat_paged_workspace_bytes(B, Hq, Hkv, Lq, max_pages, d)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    if spin_limit is not None:
        expired = ctypes.c_int(0)
        _check(lib().attnqat_debug_fwd_infer_paged(_ptr(q), B, Hq, Hkv, Lq, d, int(causal), BF16, _ptr(cache), int(num_pages),
                                                   _ptr(page_table), max_pages, _ptr(kv_lens), _ptr(o), _ptr(lse), _ptr(workspace),
                                                   workspace.numel(), _stream(), int(spin_limit), ctypes.addressof(expired)))
        return o, lse, bool(expired.value)
    _check(lib().attnqat_fwd_infer_paged(_ptr(q), B, Hq, Hkv, Lq, d, int(causal), BF16, _ptr(cache), int(num_pages),
                                         _ptr(page_table), max_pages, _ptr(kv_lens),
                                         _ptr(o), _ptr(lse), _ptr(workspace), workspace.numel(), _stream()))
    return o, lse


# The calls of a serving step.  The smallest of them take a few microseconds, of which the checks of their arguments are a good part: what is
# expected is asked for in one expression, and only where that fails is it found out which tensor it was.
_BF, _I32, _I64, _U8, _F32 = torch.bfloat16, torch.int32, torch.int64, torch.uint8, torch.float32
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _serve_refuse(ints, rows=(), cache=None):
    """Names the tensor that is not as it should be: ``ints`` (name, tensor, shape, dtype), ``rows`` (name, tensor, shape)."""
    for name, t, shape, dtype in ints:
        if not (t.is_cuda and t.dtype is dtype and t.is_contiguous() and t.shape == shape):
            raise AttnQatError(f"{name} must be a contiguous {dtype} CUDA tensor of shape {shape}")
    for name, t, shape in rows:
        if not (t.is_cuda and t.dtype is _BF and t.dim() == 3 and t.shape == shape and (t.stride(2) == 1 or t.numel() == 0)):
            raise AttnQatError(f"{name} must be a bf16 CUDA tensor [T,heads,d] of shape {tuple(shape)}, d innermost")
    if cache is not None and not (cache.is_cuda and cache.dtype is _U8 and cache.is_contiguous()):
        raise AttnQatError("cache must be a contiguous uint8 CUDA tensor")
    raise AttnQatError(f"all tensors must be on the current device (cuda:{_current_device()})")


def _serve_pages(cache, num_pages, Hkv, d):
    page = Hkv * d * 144                          # (2 parts of 128 positions of d / 2 + d / 16 bytes; the library refuses other d)
    have = cache.numel() // page if page > 0 else 0
    if num_pages is None:
        return have
    if not 0 < num_pages <= have:
        raise AttnQatError(f"cache has room for {have} pages, not for {num_pages}")
    return int(num_pages)


def page_plan_workspace_bytes(B: int) -> int:
    return lib().attnqat_page_plan_workspace_bytes(B)


def attnqat_page_plan(kv_lens, new_lens, page_table, capacity: int, free=None, workspace=None, out=None):
    """Page table, slots and positions of a serving step.  kv_lens, new_lens int32 [B]: positions that the requests have and want;
    page_table int32 [B,max_pages], updated in place; ``capacity`` the most new positions of the step; ``free`` = (free_pages int32 [places],
    free_state int32 [>= 2]: place of the first free page, number of free pages), a ring from which pages are taken and to which they are given
    back (updated in place; as many places as the cache has pages are always enough), or None for a table that is complete already.  Returns (kv_lens int32 [B], cu_q int32 [B+1], slots int64 [capacity],
    positions int32 [capacity], free_state int32 [3]: first free place, free pages, refused requests, or None without ``free``).  ``out``: those
    five; the first and the last may be kv_lens and a free_state of 3."""
    B, T, dev = kv_lens.numel(), int(capacity), kv_lens.get_device()
    if page_table.dim() != 2:
        raise AttnQatError("page_table must be [B,max_pages]")
    if T < 0:
        raise AttnQatError("capacity must not be negative")
    most = page_table.shape[1]
    ring, state = (None, None) if free is None else free
    if out is None:
        e = lambda n, t=_I32: torch.empty(n, dtype=t, device=kv_lens.device)  # noqa: E731
        out = (e(B), e(B + 1), e(T, _I64), e(T), e(3) if free is not None else None)
    lens, cu, slots, positions, state_out = out
    if not (dev == _current_device() == new_lens.get_device() == page_table.get_device() == lens.get_device() == cu.get_device() == slots.get_device() == positions.get_device()
            and kv_lens.dtype is new_lens.dtype is page_table.dtype is lens.dtype is cu.dtype is positions.dtype is _I32 and slots.dtype is _I64
            and kv_lens.shape == new_lens.shape == lens.shape == (B,) and cu.shape == (B + 1,) and slots.shape == positions.shape == (T,) and page_table.shape[0] == B
            and kv_lens.is_contiguous() and new_lens.is_contiguous() and page_table.is_contiguous() and lens.is_contiguous() and cu.is_contiguous()
            and slots.is_contiguous() and positions.is_contiguous()):
        _serve_refuse([("kv_lens", kv_lens, (B,), _I32), ("new_lens", new_lens, (B,), _I32), ("page_table", page_table, (B, most), _I32), ("out[0]", lens, (B,), _I32),
                       ("out[1]", cu, (B + 1,), _I32), ("out[2]", slots, (T,), _I64), ("out[3]", positions, (T,), _I32)])
    if free is None:
        places, state_out = 0, None
        pr = ps = po = None
    else:
        places = ring.numel()
        if not (dev == ring.get_device() == state.get_device() == state_out.get_device() and ring.dtype is state.dtype is state_out.dtype is _I32 and ring.dim() == state.dim() == 1
                and state.numel() >= 2 and state_out.shape == (3,) and ring.is_contiguous() and state.is_contiguous() and state_out.is_contiguous()):
            _serve_refuse([("free_pages", ring, (places,), _I32), ("free_state", state, (max(2, state.numel()),), _I32), ("out[4]", state_out, (3,), _I32)])
        pr, ps, po = ring.data_ptr(), state.data_ptr(), state_out.data_ptr()
    if workspace is None:
        workspace = torch.empty(max(page_plan_workspace_bytes(B), 1), dtype=_U8, device=kv_lens.device)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise AttnQatError("workspace must be contiguous, on the device of the other tensors")
    rc = (_lib or lib()).attnqat_page_plan(kv_lens.data_ptr(), new_lens.data_ptr(), B, page_table.data_ptr(), most, pr, places, ps, T, lens.data_ptr(), cu.data_ptr(),
                                           slots.data_ptr(), positions.data_ptr(), po, workspace.data_ptr(), workspace.nbytes, _stream_on(dev))
    if rc:
        _check(rc)
    return lens, cu, slots, positions, state_out


def attnqat_kv_cache_append(k, v, cache, slots, num_pages=None):
    """Quantize row t of k, v [T,Hkv,d] bf16 (any stride per row and head) into slot ``slots[t]`` (int64 [T], page * 128 + position within the page; slots
    outside the cache are left out) of the NVFP4 KV ``cache`` (uint8 CUDA tensor)."""
    shape, dev = k.shape, k.get_device()
    if not (len(shape) == 3 and v.shape == shape and k.dtype is v.dtype is _BF and slots.dtype is _I64 and slots.shape == shape[:1] and cache.dtype is _U8
            and dev == _current_device() == v.get_device() == cache.get_device() == slots.get_device() and cache.is_contiguous() and slots.is_contiguous()):
        _serve_refuse([("slots", slots, tuple(shape[:1]), _I64)], [("k", k, shape), ("v", v, shape)], cache)
    T, Hkv, d = shape
    (kt, kh, k1), (vt, vh, v1) = k.stride(), v.stride()
    if not k1 == v1 == 1 and k.numel() > 0:
        _serve_refuse([], [("k", k, shape), ("v", v, shape)])
    rc = (_lib or lib()).attnqat_kv_cache_append(k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, T, Hkv, d, BF16, cache.data_ptr(), _serve_pages(cache, num_pages, Hkv, d),
                                                 slots.data_ptr(), _stream_on(dev))
    if rc:
        _check(rc)


def attnqat_kv_cache_read(cache, slots, Hkv: int, d: int, num_pages=None, out=None):
    """The values that the NVFP4 KV ``cache`` holds in ``slots`` (int64 [T]; zeros for a slot outside the cache).  Returns (k, v) bf16
    [T,Hkv,d]; ``out``: those two, of any stride per row and head."""
    T, dev = slots.numel(), slots.get_device()
    shape = (T, Hkv, d)
    k, v = out if out is not None else tuple(torch.empty(shape, dtype=_BF, device=cache.device) for _ in range(2))
    if not (k.shape == v.shape == shape and k.dtype is v.dtype is _BF and slots.dtype is _I64 and slots.dim() == 1 and cache.dtype is _U8
            and dev == _current_device() == k.get_device() == v.get_device() == cache.get_device() and cache.is_contiguous() and slots.is_contiguous()):
        _serve_refuse([("slots", slots, (T,), _I64)], [("out[0]", k, shape), ("out[1]", v, shape)], cache)
    (kt, kh, k1), (vt, vh, v1) = k.stride(), v.stride()
    if not k1 == v1 == 1 and k.numel() > 0:
        _serve_refuse([], [("out[0]", k, shape), ("out[1]", v, shape)])
    rc = (_lib or lib()).attnqat_kv_cache_read(cache.data_ptr(), _serve_pages(cache, num_pages, Hkv, d), slots.data_ptr(), T, Hkv, d, BF16, k.data_ptr(), kt, kh,
                                               v.data_ptr(), vt, vh, _stream_on(dev))
    if rc:
        _check(rc)
    return k, v


def _within_int(x):
    """The nearest number that the library's int holds: ctypes would take the low 32 bits.  (For numbers that are limits: more rows than there are, a window
    beyond every length, anything below 1.)"""
    return max(-1, min(int(x), 0x7FFFFFFF))


def kv4_ragged_workspace_bytes(T: int, B: int, Hq: int, Hkv: int, max_q: int, max_pages: int, d: int) -> int:
    return lib().attnqat_kv4_ragged_workspace_bytes(T, B, Hq, Hkv, _within_int(max_q), max_pages, d)


def attnqat_fwd_kv4_ragged(q, cu_q, cache, num_pages, page_table, kv_lens, Hkv: int, causal: bool, max_q=None, window: int = 0, scale=None,
                           workspace=None, out=None):
    """Attention over an NVFP4 KV cache, Q and the probabilities not quantized, of sequences with different numbers of queries.  q [T,Hq,d] bf16 (any stride
    per row and head), rows cu_q[b] .. cu_q[b+1]-1 (int32 [B+1]) being the last positions of sequence b, which has kv_lens[b] keys (int32 [B]) in the
    pages page_table[b] (int32 [B,max_pages]).  ``max_q``: the most rows of a sequence (default T; the
    kernels are chosen by it, and a decode step that does not say 1 pays for those of many rows); ``window`` (causal only): a row sees that many keys at
    most, its own position included; ``scale``: default 1/sqrt(d).  Returns (o bf16 [T,Hq,d], lse fp32 [T,Hq]); ``out``: those two (lse may be None)."""
    shape, dev, B = q.shape, q.get_device(), kv_lens.numel()
    if len(shape) != 3 or page_table.dim() != 2:
        raise AttnQatError("q must be [T,Hq,d] and page_table [B,max_pages]")
    T, Hq, d = shape
    most = page_table.shape[1]
    o, lse = out if out is not None else (torch.empty(shape, dtype=_BF, device=q.device), torch.empty((T, Hq), dtype=_F32, device=q.device))
    if not (q.dtype is o.dtype is _BF and o.shape == shape and kv_lens.dtype is cu_q.dtype is page_table.dtype is _I32 and cache.dtype is _U8
            and kv_lens.shape == (B,) and cu_q.shape == (B + 1,) and page_table.shape[0] == B
            and dev == _current_device() == o.get_device() == cu_q.get_device() == cache.get_device() == page_table.get_device() == kv_lens.get_device()
            and cache.is_contiguous() and cu_q.is_contiguous() and page_table.is_contiguous() and kv_lens.is_contiguous()
            and (lse is None or (lse.dtype is _F32 and lse.shape == (T, Hq) and lse.get_device() == dev and lse.is_contiguous()))):
        _serve_refuse([("kv_lens", kv_lens, (B,), _I32), ("cu_q", cu_q, (B + 1,), _I32), ("page_table", page_table, (B, most), _I32)]
                      + ([] if lse is None else [("out[1]", lse, (T, Hq), _F32)]), [("q", q, shape), ("out[0]", o, shape)], cache)
    (qt, qh, q1), (ot, oh, o1) = q.stride(), o.stride()
    if not q1 == o1 == 1 and q.numel() > 0:
        _serve_refuse([], [("q", q, shape), ("out[0]", o, shape)])
    max_q, window = max(T, 1) if max_q is None else _within_int(max_q), _within_int(window)
    if workspace is None:
        workspace = torch.empty(max(kv4_ragged_workspace_bytes(T, B, Hq, Hkv, max_q, most, d), 1), dtype=_U8, device=q.device)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise AttnQatError("workspace must be contiguous, on the device of the other tensors")
    rc = (_lib or lib()).attnqat_fwd_kv4_ragged(q.data_ptr(), qt, qh, cu_q.data_ptr(), T, max_q, B, Hq, Hkv, d, 1 if causal else 0, window, d ** -0.5 if scale is None else scale, BF16,
                                                cache.data_ptr(), _serve_pages(cache, num_pages, Hkv, d), page_table.data_ptr(), most, kv_lens.data_ptr(),
                                                o.data_ptr(), ot, oh, None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes, _stream_on(dev))
    if rc:
        _check(rc)
    return o, lse


ROPE_PAIRED, ROPE_HALVES = 0, 1


class Rope(ctypes.Structure):
    """How the values of a head turn with their positions (host memory; made by ``rope_table``)."""
    _fields_ = [("pairs", ctypes.c_int), ("axes", ctypes.c_int), ("layout", ctypes.c_int), ("reserved", ctypes.c_int),
                ("turns", ctypes.c_uint64 * 64), ("axis", ctypes.c_uint32 * 4)]


def rope_table(dims, theta: float = 10000.0, layout: str = "paired", freqs=None, axis=None) -> Rope:
    """A table of rotary positions, to be kept by the program.  ``dims``: how many values of a head turn with each axis, e.g. (128,) or, for time, height and
    width, (44, 42, 42): pair i of an axis of n values turns by theta^(-2i/n) radians per position, from i = 0 in every axis, as video models have it.
    ``layout``: "paired" (elements 2i, 2i+1) or "halves" (i and i + half the turned values).  ``freqs`` and ``axis``: radians per position and axis of every
    pair where they follow another rule (of ``dims`` the number of axes and of values is left, and its sections where ``axis`` is not given).  A language model whose
    axes share one ladder of frequencies over the head, cut into sections, has ``rope_table((32, 48, 48), layout="halves", freqs=[theta ** (-2.0 * i / 128) for i in range(64)])``."""
    dims = tuple(int(n) for n in dims)
    if layout not in ("paired", "halves"):
        raise AttnQatError("layout must be 'paired' or 'halves'")
    if not 1 <= len(dims) <= 4 or any(n < 0 or n % 2 for n in dims) or not 2 <= sum(dims) <= 128:
        raise AttnQatError("dims must be one to four even numbers, of 2 to 128 values together")
    pairs = sum(dims) // 2
    if freqs is None:
        freqs = [float(theta) ** (-2.0 * i / n) for n in dims for i in range(n // 2)]
    if axis is None:
        axis = [a for a, n in enumerate(dims) for _ in range(n // 2)]
    freqs, axis = [float(f) for f in freqs], [int(a) for a in axis]
    if len(freqs) != pairs or len(axis) != pairs or any(not 0 <= a < len(dims) for a in axis):
        raise AttnQatError(f"freqs and axis must have an entry for each of the {pairs} pairs, axis below {len(dims)}")
    rope = Rope()
    _check(lib().attnqat_rope_table(ctypes.addressof(rope), pairs, len(dims), ROPE_HALVES if layout == "halves" else ROPE_PAIRED, (ctypes.c_double * pairs)(*freqs), (ctypes.c_uint8 * pairs)(*axis)))
    return rope


def _rope_refuse(q, k, positions, rope, out):
    """Names what is not as it should be."""
    if not isinstance(rope, Rope):
        raise AttnQatError("rope must be a table made by rope_table")
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        raise AttnQatError("q and k must be [B,heads,L,d]")
    (B, _, L, d), dev = q.shape, q.get_device()
    if not (positions.dtype is _I32 and positions.is_cuda and positions.is_contiguous() and positions.shape in ((L, rope.axes), (B, L, rope.axes))):
        raise AttnQatError(f"positions must be a contiguous int32 CUDA tensor [{L},{rope.axes}] or [{B},{L},{rope.axes}]")
    for name, t, o in (("q", q, out[0]), ("k", k, out[1])):
        for x in () if t is None else (t, o):
            if not (x is not None and x.is_cuda and x.dtype is _BF and x.shape == (B, t.shape[1], L, d) and (x.stride(3) == 1 or x.numel() == 0)):
                raise AttnQatError(f"{name} and its output must be bf16 CUDA tensors {(B, t.shape[1], L, d)}, d innermost")
    raise AttnQatError(f"all tensors must be on the current device (cuda:{_current_device()})")


def _rope_call(f, q, k, positions, rope, out):
    if out is None:
        out = (torch.empty(q.shape, dtype=_BF, device=q.device), None if k is None else torch.empty(k.shape, dtype=_BF, device=q.device))
    qo, ko = out
    dev, shape, at = q.get_device(), q.shape, positions.shape
    if not (type(rope) is Rope and len(shape) == 4 and q.dtype is qo.dtype is _BF and positions.dtype is _I32 and qo.shape == shape and positions.is_contiguous()
            and dev == _current_device() == qo.get_device() == positions.get_device()):
        _rope_refuse(q, k, positions, rope, out)
    B, Hq, L, d = shape
    axes = rope.axes
    (qb, qh, qt, q1), (ob, oh, ot, o1) = q.stride(), qo.stride()
    if not (q1 == o1 == 1 or q.numel() == 0) or not (at == (L, axes) or at == (B, L, axes)):
        _rope_refuse(q, k, positions, rope, out)
    if k is None:
        Hkv, kp, kb, kh, kt, kop, kob, koh, kot = 0, None, 0, 0, 0, None, 0, 0, 0
    else:
        ks = k.shape
        if not (len(ks) == 4 and ko is not None and ko.shape == ks and k.dtype is ko.dtype is _BF and ks[0] == B and ks[2:] == shape[2:] and dev == k.get_device() == ko.get_device()):
            _rope_refuse(q, k, positions, rope, out)
        (kb, kh, kt, k1), (kob, koh, kot, ko1) = k.stride(), ko.stride()
        if not (k1 == ko1 == 1 or k.numel() == 0):
            _rope_refuse(q, k, positions, rope, out)
        Hkv, kp, kop = ks[1], k.data_ptr(), ko.data_ptr()
    rc = f(q.data_ptr(), qb, qh, qt, kp, kb, kh, kt, B, Hq, Hkv, L, d, BF16, positions.data_ptr(), L * axes if len(at) == 3 else 0, ctypes.addressof(rope),
           qo.data_ptr(), ob, oh, ot, kop, kob, koh, kot, _stream_on(dev))
    if rc:
        _check(rc)
    return out


def attnqat_rope_fwd(q, k, positions, rope, out=None):
    """Rotary positions of q [B,Hq,L,d] and k [B,Hkv,L,d] (bf16, any stride per batch, head and token, d innermost; k may be None).  positions int32 [L,axes], or
    [B,L,axes]; ``rope``: ``rope_table``.  Returns (q, k), contiguous: what attnqat_fwd takes; ``out``: those two, of any strides, each of which may be its input."""
    return _rope_call((_lib or lib()).attnqat_rope_fwd, q, k, positions, rope, out)


def attnqat_rope_bwd(dq, dk, positions, rope, out=None):
    """Gradient of attnqat_rope_fwd: from dq [B,Hq,L,d] and dk [B,Hkv,L,d] of its outputs to those of its inputs.  Arguments as there; ``out`` may be views of one
    projection's gradient."""
    return _rope_call((_lib or lib()).attnqat_rope_bwd, dq, dk, positions, rope, out)


def attnqat_kv_cache_append_rope(q, k, v, positions, rope, cache, slots, num_pages=None, out=None):
    """attnqat_kv_cache_append with rotary positions on the way: k turned, rounded to bf16 and quantized, v as it is, and q [T,Hq,d] (or None) turned.  positions
    int32 [T,axes], or [T] with one axis; ``rope``: ``rope_table``.  Returns the turned q, bf16 [T,Hq,d]; ``out``: that, of any stride per row and head, or q itself."""
    shape, dev = k.shape, k.get_device()
    if not isinstance(rope, Rope):
        raise AttnQatError("rope must be a table made by rope_table")
    if not (len(shape) == 3 and v.shape == shape and k.dtype is v.dtype is _BF and slots.dtype is _I64 and slots.shape == shape[:1] and cache.dtype is _U8
            and positions.dtype is _I32 and positions.is_contiguous() and (positions.shape == (shape[0], rope.axes) or (rope.axes == 1 and positions.shape == shape[:1]))
            and dev == _current_device() == v.get_device() == cache.get_device() == slots.get_device() == positions.get_device() and cache.is_contiguous() and slots.is_contiguous()):
        _serve_refuse([("slots", slots, tuple(shape[:1]), _I64), ("positions", positions, (shape[0], rope.axes), _I32)], [("k", k, shape), ("v", v, shape)], cache)
    T, Hkv, d = shape
    (kt, kh, k1), (vt, vh, v1) = k.stride(), v.stride()
    if not k1 == v1 == 1 and k.numel() > 0:
        _serve_refuse([], [("k", k, shape), ("v", v, shape)])
    Hq, qp, qt, qh, op, ot, oh = 0, None, 0, 0, None, 0, 0
    if q is not None:
        if q.dim() != 3:
            raise AttnQatError("q must be [T,Hq,d]")
        Hq = q.shape[1]
        if out is None:
            out = torch.empty((T, Hq, d), dtype=_BF, device=q.device)
        (qt, qh, q1), want = q.stride(), (T, Hq, d)
        if not (q.shape == out.shape == want and q.dtype is out.dtype is _BF and dev == q.get_device() == out.get_device() and (q1 == out.stride(2) == 1 or q.numel() == 0)):
            _serve_refuse([], [("q", q, want), ("out", out, want)])
        ot, oh, _ = out.stride()
        qp, op = q.data_ptr(), out.data_ptr()
    rc = (_lib or lib()).attnqat_kv_cache_append_rope(qp, qt, qh, k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, T, Hq, Hkv, d, BF16, positions.data_ptr(), ctypes.addressof(rope),
                                                      cache.data_ptr(), _serve_pages(cache, num_pages, Hkv, d), slots.data_ptr(), op, ot, oh, _stream_on(dev))
    if rc:
        _check(rc)
    return out if q is not None else None


def kv_summary_page_bytes(Hkv: int, d: int) -> int:
    return lib().attnqat_kv_summary_page_bytes(Hkv, d)


def _summary_pages(summary, pages, Hkv, d):
    if pages < 1 or summary.numel() < pages * Hkv * (d + 16):
        raise AttnQatError(f"summary has no room for {pages} pages (of 1 at least)")


def attnqat_kv_summarize(cache, slots, summary, Hkv: int, d: int, num_pages=None):
    """The means of the keys of every page whose last position is among ``slots`` (int64 [T], those that have just been appended), in 8 bits, into ``summary``
    (uint8 CUDA tensor of num_pages * kv_summary_page_bytes(Hkv, d) bytes)."""
    dev = slots.get_device()
    if not (slots.dtype is _I64 and slots.dim() == 1 and cache.dtype is summary.dtype is _U8 and dev == _current_device() == cache.get_device() == summary.get_device()
            and cache.is_contiguous() and summary.is_contiguous() and slots.is_contiguous()):
        _serve_refuse([("slots", slots, (slots.numel(),), _I64), ("summary", summary, (summary.numel(),), _U8)], (), cache)
    pages = _serve_pages(cache, num_pages, Hkv, d)
    _summary_pages(summary, pages, Hkv, d)
    rc = (_lib or lib()).attnqat_kv_summarize(cache.data_ptr(), pages, slots.data_ptr(), slots.numel(), Hkv, d, summary.data_ptr(), _stream_on(dev))
    if rc:
        _check(rc)


def attnqat_kv_select(q, cu_q, summary, num_pages: int, page_table, kv_lens, Hkv: int, n_blocks: int, first: int = 1, last: int = 1, max_q=None, out=None):
    """The pages that every row attends to: its sequence's ``first`` first ones, ``last`` last ones (its own among them), and those whose keys' mean
    (``attnqat_kv_summarize``) gives the highest score, ``n_blocks`` at most.  q (turned), cu_q, page_table, kv_lens: as for attnqat_fwd_kv4_ragged.  max_q: the most rows of a
    sequence, by which the work is laid out (T where left out; the choice is the same with any).  A step of single tokens says 1.  Returns int32 [T,Hkv,n_blocks]: page numbers
    of the sequence, ascending, -1 behind them; ``out``: that."""
    shape, dev, B = q.shape, q.get_device(), kv_lens.numel()
    if len(shape) != 3 or page_table.dim() != 2:
        raise AttnQatError("q must be [T,Hq,d] and page_table [B,max_pages]")
    T, Hq, d = shape
    most, want = page_table.shape[1], (T, Hkv, n_blocks)
    if out is None:
        out = torch.empty((T, max(Hkv, 0), max(n_blocks, 0)), dtype=_I32, device=q.device)
    (qt, qh, q1) = q.stride()
    if not (q.dtype is _BF and (q1 == 1 or q.numel() == 0) and kv_lens.dtype is cu_q.dtype is page_table.dtype is out.dtype is _I32 and summary.dtype is _U8 and out.shape == want
            and kv_lens.shape == (B,) and cu_q.shape == (B + 1,) and page_table.shape[0] == B
            and dev == _current_device() == cu_q.get_device() == summary.get_device() == page_table.get_device() == kv_lens.get_device() == out.get_device()
            and summary.is_contiguous() and cu_q.is_contiguous() and page_table.is_contiguous() and kv_lens.is_contiguous() and out.is_contiguous()):
        _serve_refuse([("kv_lens", kv_lens, (B,), _I32), ("cu_q", cu_q, (B + 1,), _I32), ("page_table", page_table, (B, most), _I32), ("out", out, want, _I32),
                       ("summary", summary, (summary.numel(),), _U8)], [("q", q, shape)])
    _summary_pages(summary, num_pages, Hkv, d)
    rc = (_lib or lib()).attnqat_kv_select(q.data_ptr(), qt, qh, cu_q.data_ptr(), T, max(T, 1) if max_q is None else _within_int(max_q), B, Hq, Hkv, d, BF16, summary.data_ptr(),
                                           num_pages, page_table.data_ptr(), most, kv_lens.data_ptr(), n_blocks, _within_int(first), _within_int(last), out.data_ptr(), _stream_on(dev))
    if rc:
        _check(rc)
    return out


def kv4_sparse_workspace_bytes(T: int, Hq: int, Hkv: int, max_q: int, n_blocks: int, d: int) -> int:
    return lib().attnqat_kv4_sparse_workspace_bytes(T, Hq, Hkv, _within_int(max_q), n_blocks, d)


def attnqat_fwd_kv4_sparse(q, cu_q, cache, num_pages, page_table, kv_lens, Hkv: int, blocks, max_q=None, scale=None, workspace=None, out=None):
    """attnqat_fwd_kv4_ragged (causal) over a choice of pages: row t of kv head h sees those of its keys that lie in pages ``blocks[t,h]`` of its sequence (int32
    [T,Hkv,n_blocks], from attnqat_kv_select or any other; entries outside the row's pages are passed over).  Other arguments, and (o, lse), as there.

    max_q: the most rows of a sequence, the same number as for the workspace.  Where it is left out it is T, which is right and lays the work out for long pieces: rows of up to
    16 * Hkv / Hq sequences share a workgroup, each going through the pages of all.  A step of single tokens says 1, one of drafted tokens their number.  The order of the sums
    follows from it, and with that the last bits."""
    shape, dev, B = q.shape, q.get_device(), kv_lens.numel()
    if len(shape) != 3 or page_table.dim() != 2 or blocks.dim() != 3:
        raise AttnQatError("q must be [T,Hq,d], page_table [B,max_pages] and blocks [T,Hkv,n_blocks]")
    T, Hq, d = shape
    most, n_blocks = page_table.shape[1], blocks.shape[2]
    o, lse = out if out is not None else (torch.empty(shape, dtype=_BF, device=q.device), torch.empty((T, Hq), dtype=_F32, device=q.device))
    if not (q.dtype is o.dtype is _BF and o.shape == shape and kv_lens.dtype is cu_q.dtype is page_table.dtype is blocks.dtype is _I32 and cache.dtype is _U8
            and kv_lens.shape == (B,) and cu_q.shape == (B + 1,) and page_table.shape[0] == B and blocks.shape[:2] == (T, Hkv)
            and dev == _current_device() == o.get_device() == cu_q.get_device() == cache.get_device() == page_table.get_device() == kv_lens.get_device() == blocks.get_device()
            and cache.is_contiguous() and cu_q.is_contiguous() and page_table.is_contiguous() and kv_lens.is_contiguous() and blocks.is_contiguous()
            and (lse is None or (lse.dtype is _F32 and lse.shape == (T, Hq) and lse.get_device() == dev and lse.is_contiguous()))):
        _serve_refuse([("kv_lens", kv_lens, (B,), _I32), ("cu_q", cu_q, (B + 1,), _I32), ("page_table", page_table, (B, most), _I32), ("blocks", blocks, (T, Hkv, n_blocks), _I32)]
                      + ([] if lse is None else [("out[1]", lse, (T, Hq), _F32)]), [("q", q, shape), ("out[0]", o, shape)], cache)
    (qt, qh, q1), (ot, oh, o1) = q.stride(), o.stride()
    if not q1 == o1 == 1 and q.numel() > 0:
        _serve_refuse([], [("q", q, shape), ("out[0]", o, shape)])
    max_q = max(T, 1) if max_q is None else _within_int(max_q)
    if workspace is None:
        workspace = torch.empty(max(kv4_sparse_workspace_bytes(T, Hq, Hkv, max_q, n_blocks, d), 1), dtype=_U8, device=q.device)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise AttnQatError("workspace must be contiguous, on the device of the other tensors")
    rc = (_lib or lib()).attnqat_fwd_kv4_sparse(q.data_ptr(), qt, qh, cu_q.data_ptr(), T, max_q, B, Hq, Hkv, d, d ** -0.5 if scale is None else scale, BF16, cache.data_ptr(),
                                                _serve_pages(cache, num_pages, Hkv, d), page_table.data_ptr(), most, kv_lens.data_ptr(), blocks.data_ptr(), n_blocks,
                                                o.data_ptr(), ot, oh, None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes, _stream_on(dev))
    if rc:
        _check(rc)
    return o, lse


def attnqat_debug_fwd_p_opt(q, k, v, causal: bool, row0: int, options: int):
    """attnqat_debug_fwd_p with the option bits of attnqat_fwd_opt."""
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    o = torch.empty_like(q)
    lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
    p = torch.zeros((B, Hq, 128, L), dtype=torch.float32, device=q.device)
    ws, nb = _workspace(WS_FWD, B, Hq, Hkv, L, d, None)
    _check(lib().attnqat_debug_fwd_p_opt(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, L, d, int(causal), BF16, int(options),
                                         _ptr(o), _ptr(lse), row0, _ptr(p), _ptr(ws), nb, _stream()))
    return o, lse, p


def attnqat_debug_bwd_p(q, k, v, d_o, lse, o_hp, causal: bool, row0: int):
    """attnqat_bwd that also returns P^F (the re-quantized recomputed P of Alg. 3) of query rows [row0, row0+128):
    (dq, dk, dv, p [B,Hq,128,L] fp32)."""
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    p = torch.zeros((B, Hq, 128, L), dtype=torch.float32, device=q.device)
    ws, nb = _workspace(WS_BWD, B, Hq, Hkv, L, d, None)
    _check(lib().attnqat_debug_bwd_p(_ptr(q), _ptr(k), _ptr(v), _ptr(d_o), _ptr(lse), _ptr(o_hp), B, Hq, Hkv, L, d, int(causal), BF16,
                                     _ptr(dq), _ptr(dk), _ptr(dv), int(row0), _ptr(p), _ptr(ws), nb, _stream()))
    return dq, dk, dv, p


def attnqat_fwd_opt(q, k, v, causal: bool, options: int, train: bool = True, workspace=None, out=None):
    """Alg. 2 (train) or Alg. 1 with the option bits of Sec. 3.2 (OPT_SMOOTH_K).  Returns (o, lse, o_hp or None)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _dev_bf16(t, n)
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
        o_hp = torch.empty((B, Hq, L, d), dtype=torch.float32, device=q.device) if train else None
    else:
        o, lse, o_hp = out
    ws, nb = _workspace(WS_FWD, B, Hq, Hkv, L, d, workspace)
    _check(lib().attnqat_fwd_opt(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, L, d, int(causal), BF16, int(options),
                                 _ptr(o), _ptr(lse), _ptr(o_hp), _ptr(ws), nb, _stream()))
    return o, lse, o_hp


def attnqat_bwd_opt(q, k, v, d_o, lse, o_hp, causal: bool, options: int, workspace=None, out=None):
    """Alg. 3 with the same option bits as the forward.  Returns (dq, dk, dv) bf16."""
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (d_o, "d_o")):
        _dev_bf16(t, n)
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    if out is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    else:
        dq, dk, dv = out
    ws, nb = _workspace(WS_BWD, B, Hq, Hkv, L, d, workspace)
    _check(lib().attnqat_bwd_opt(_ptr(q), _ptr(k), _ptr(v), _ptr(d_o), _ptr(lse), _ptr(o_hp),
                                 B, Hq, Hkv, L, d, int(causal), BF16, int(options),
                                 _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), nb, _stream()))
    return dq, dk, dv


def attnqat_fwd_mx(q, k, v, causal: bool, workspace=None, out=None):
    """Alg. 2 in the MX format (16-bit matrix path).  Returns (o bf16, lse fp32 [B,Hq,L], o_hp fp32)."""
    return attnqat_fwd(q, k, v, causal, workspace, out, _mx=True)


def attnqat_bwd_mx(q, k, v, d_o, lse, o_hp, causal: bool, workspace=None, out=None):
    """Alg. 3 in the MX format.  Returns (dq, dk, dv) bf16."""
    return attnqat_bwd(q, k, v, d_o, lse, o_hp, causal, workspace, out, _mx=True)


def attnqat_fwd(q, k, v, causal: bool, workspace=None, out=None, _mx=False):
    """Alg. 2.  Returns (o bf16, lse fp32 [B,Hq,L], o_hp fp32)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _dev_bf16(t, n)
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
        o_hp = torch.empty((B, Hq, L, d), dtype=torch.float32, device=q.device)
    else:
        o, lse, o_hp = out
    ws, nb = _workspace(WS_FWD_MX if _mx else WS_FWD, B, Hq, Hkv, L, d, workspace)
    _check((lib().attnqat_fwd_mx if _mx else lib().attnqat_fwd)(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, L, d, int(causal), BF16,
                             _ptr(o), _ptr(lse), _ptr(o_hp), _ptr(ws), nb, _stream()))
    return o, lse, o_hp


def attnqat_fwd_infer(q, k, v, causal: bool, workspace=None, out=None):
    """Alg. 1.  Returns (o bf16, lse fp32)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _dev_bf16(t, n)
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
    else:
        o, lse = out
    ws, nb = _workspace(WS_FWD_INFER, B, Hq, Hkv, L, d, workspace)
    _check(lib().attnqat_fwd_infer(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, L, d, int(causal), BF16,
                                   _ptr(o), _ptr(lse), _ptr(ws), nb, _stream()))
    return o, lse


def attnqat_fwd_infer_bf16pv(q, k, v, causal: bool, workspace=None, out=None):
    """Alg. 1 in the mixed recipe of Sec. 2.5: NVFP4 Q K^T, P-tilde and V in bf16.  Returns (o bf16, lse fp32)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _dev_bf16(t, n)
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
    else:
        o, lse = out
    ws, nb = _workspace(WS_FWD_INFER, B, Hq, Hkv, L, d, workspace)
    _check(lib().attnqat_fwd_infer_bf16pv(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, L, d, int(causal), BF16,
                                          _ptr(o), _ptr(lse), _ptr(ws), nb, _stream()))
    return o, lse


def attnqat_fwd_infer_static(q, k, v, causal: bool, out):
    """attnqat_fwd_infer on the library's static scratch array: allocates nothing, so the outputs (o bf16, lse fp32)
    must be passed in.  Raises for problems that need more than STATIC_SCRATCH_BYTES of scratch."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _dev_bf16(t, n)
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    o, lse = out
    _check(lib().attnqat_fwd_infer_static(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, L, d, int(causal), BF16,
                                          _ptr(o), _ptr(lse), _stream()))
    return o, lse


def attnqat_fwd_infer_packed(qp, kp, vp, causal: bool, d: int, workspace=None, out=None):
    """Alg. 1 on already quantized tensors: qp, kp, vp are (codes, scales) pairs from attnqat_quantize.
    Returns (o bf16, lse fp32), bit-identical to attnqat_fwd_infer on the tensors the codes came from."""
    (qc, qs), (kc, ks), (vc, vs) = qp, kp, vp
    B, Hq, L, _ = qc.shape
    Hkv = kc.shape[1]
    if out is None:
        o = torch.empty((B, Hq, L, d), dtype=torch.bfloat16, device=qc.device)
        lse = torch.empty((B, Hq, L), dtype=torch.float32, device=qc.device)
    else:
        o, lse = out
    ws, nb = _workspace(WS_FWD_INFER, B, Hq, Hkv, L, d, workspace)
    _check(lib().attnqat_fwd_infer_packed(_ptr(qc), _ptr(qs), _ptr(kc), _ptr(ks), _ptr(vc), _ptr(vs), B, Hq, Hkv, L, d,
                                          int(causal), BF16, _ptr(o), _ptr(lse), _ptr(ws), nb, _stream()))
    return o, lse


def attnqat_bwd_packed(qp, kp, vp, d_o, lse, o_hp, causal: bool, workspace=None, out=None):
    """Alg. 3 from the saved quantized Q, K, V of the forward ((codes, scales) pairs).  Returns (dq, dk, dv) bf16."""
    (qc, qs), (kc, ks), (vc, vs) = qp, kp, vp
    _dev_bf16(d_o, "d_o")
    B, Hq, L, d = d_o.shape
    Hkv = kc.shape[1]
    if out is None:
        dq = torch.empty_like(d_o)
        dk = torch.empty((B, Hkv, L, d), dtype=torch.bfloat16, device=d_o.device)
        dv = torch.empty_like(dk)
    else:
        dq, dk, dv = out
    ws, nb = _workspace(WS_BWD, B, Hq, Hkv, L, d, workspace)
    _check(lib().attnqat_bwd_packed(_ptr(qc), _ptr(qs), _ptr(kc), _ptr(ks), _ptr(vc), _ptr(vs), _ptr(d_o), _ptr(lse), _ptr(o_hp),
                                    B, Hq, Hkv, L, d, int(causal), BF16, _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), nb, _stream()))
    return dq, dk, dv


def attnqat_quantize_mx(x, axis: int = 0, want_codes=True, want_xf=True):
    """MX phi (E2M1, blocks of 32, E8M0 scale) along d (axis 0) or along the sequence (axis 1).
    Returns (codes u8, scales u8, xf bf16): axis 0 [B,H,L,d/2], [B,H,L,d/32]; axis 1 [B,H,d,Lc/2],
    [B,H,d,Lc/32] with Lc = L rounded up to 32."""
    _dev_bf16(x, "x")
    B, H, L, d = x.shape
    if axis == 0:
        cshape, sshape = (B, H, L, d // 2), (B, H, L, d // 32)
    else:
        Lc = (L + 31) // 32 * 32
        cshape, sshape = (B, H, d, Lc // 2), (B, H, d, Lc // 32)
    codes = torch.empty(cshape, dtype=torch.uint8, device=x.device) if want_codes else None
    scales = torch.empty(sshape, dtype=torch.uint8, device=x.device) if want_codes else None
    xf = torch.empty_like(x) if want_xf else None
    _check(lib().attnqat_quantize_mx(_ptr(x), B, H, L, d, BF16, int(axis), _ptr(codes), _ptr(scales), _ptr(xf), _stream()))
    return codes, scales, xf


def attnqat_quantize_mxfp8(x, want_codes=True, want_xf=True):
    """MXFP8 phi (E4M3 elements, blocks of 32 along the sequence, E8M0 scale): how V is held in the mixed recipe.
    Returns (codes u8 [B,H,d,Lc], scales u8 [B,H,d,Lc/32], xf bf16) with Lc = L rounded up to 32."""
    _dev_bf16(x, "x")
    B, H, L, d = x.shape
    Lc = (L + 31) // 32 * 32
    codes = torch.empty((B, H, d, Lc), dtype=torch.uint8, device=x.device) if want_codes else None
    scales = torch.empty((B, H, d, Lc // 32), dtype=torch.uint8, device=x.device) if want_codes else None
    xf = torch.empty_like(x) if want_xf else None
    _check(lib().attnqat_quantize_mxfp8(_ptr(x), B, H, L, d, BF16, 1, _ptr(codes), _ptr(scales), _ptr(xf), _stream()))
    return codes, scales, xf


def attnqat_fwd_infer_mx_fp8pv(q, k, v, causal: bool, workspace=None, out=None):
    """Alg. 1, mixed recipe: FP4 (MX) Q K^T, MXFP8 P V.  Returns (o bf16, lse fp32)."""
    return attnqat_fwd_infer_mx(q, k, v, causal, workspace, out, _fp8pv=True)


def attnqat_fwd_infer_mx(q, k, v, causal: bool, workspace=None, out=None, _fp8pv=False):
    """Alg. 1 in the MX format on the scaled FP4 MFMA.  Returns (o bf16, lse fp32)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _dev_bf16(t, n)
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
    else:
        o, lse = out
    ws, nb = _workspace(WS_FWD_INFER_MX_FP8PV if _fp8pv else WS_FWD_INFER_MX, B, Hq, Hkv, L, d, workspace)
    _check((lib().attnqat_fwd_infer_mx_fp8pv if _fp8pv else lib().attnqat_fwd_infer_mx)(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, L, d, int(causal), BF16,
                                      _ptr(o), _ptr(lse), _ptr(ws), nb, _stream()))
    return o, lse


def attnqat_bwd(q, k, v, d_o, lse, o_hp, causal: bool, workspace=None, out=None, _mx=False):
    """Alg. 3.  Returns (dq, dk, dv) bf16."""
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (d_o, "d_o")):
        _dev_bf16(t, n)
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    if not (lse.dtype == torch.float32 and lse.is_contiguous() and o_hp.dtype == torch.float32
            and o_hp.is_contiguous()):
        raise AttnQatError("lse and o_hp must be contiguous fp32 tensors")
    if out is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    else:
        dq, dk, dv = out
    ws, nb = _workspace(WS_BWD_MX if _mx else WS_BWD, B, Hq, Hkv, L, d, workspace)
    _check((lib().attnqat_bwd_mx if _mx else lib().attnqat_bwd)(_ptr(q), _ptr(k), _ptr(v), _ptr(d_o), _ptr(lse), _ptr(o_hp),
                             B, Hq, Hkv, L, d, int(causal), BF16,
                             _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), nb, _stream()))
    return dq, dk, dv


ABL_D_FROM_O, ABL_P_UNQUANTIZED = 1, 2


def attnqat_bwd_ablation(q, k, v, d_o, lse, o_hp, o, causal: bool, ablation: int, workspace=None, out=None):
    """Alg. 3 with the ablations of Sec. 3.2 switched on by the bit set ``ablation``
    (ABL_D_FROM_O: D from the bf16 output ``o``; ABL_P_UNQUANTIZED: dV from the fp32 P).
    Returns (dq, dk, dv) bf16."""
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (d_o, "d_o")):
        _dev_bf16(t, n)
    if ablation & ABL_D_FROM_O:
        _dev_bf16(o, "o")
    elif not (o_hp.dtype == torch.float32 and o_hp.is_contiguous()):
        raise AttnQatError("o_hp must be a contiguous fp32 tensor")
    if not (lse.dtype == torch.float32 and lse.is_contiguous()):
        raise AttnQatError("lse must be a contiguous fp32 tensor")
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    if out is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    else:
        dq, dk, dv = out
    ws, nb = _workspace(WS_BWD, B, Hq, Hkv, L, d, workspace)
    _check(lib().attnqat_bwd_ablation(_ptr(q), _ptr(k), _ptr(v), _ptr(d_o), _ptr(lse),
                                      _ptr(o_hp) if o_hp is not None else None, _ptr(o) if o is not None else None,
                                      B, Hq, Hkv, L, d, int(causal), BF16, int(ablation),
                                      _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), nb, _stream()))
    return dq, dk, dv


def attnqat_debug_fwd_p_mx(q, k, v, causal: bool, row0: int):
    """attnqat_debug_fwd_p for the MX forward of attnqat_fwd_mx."""
    return attnqat_debug_fwd_p(q, k, v, causal, row0, _mx=True)


def attnqat_debug_fwd_p(q, k, v, causal: bool, row0: int, _mx=False):
    """Test hook: (o, lse, P-tilde^F fp32 [B,Hq,128,L]) for query rows [row0, row0+128)."""
    B, Hq, L, d = q.shape
    Hkv = k.shape[1]
    o = torch.empty_like(q)
    lse = torch.empty((B, Hq, L), dtype=torch.float32, device=q.device)
    p = torch.zeros((B, Hq, 128, L), dtype=torch.float32, device=q.device)    # skipped (masked) tiles are not written
    ws, nb = _workspace(WS_FWD_MX if _mx else WS_FWD_INFER, B, Hq, Hkv, L, d, None)
    _check((lib().attnqat_debug_fwd_p_mx if _mx else lib().attnqat_debug_fwd_p)(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, L, d, int(causal), BF16,
                                     _ptr(o), _ptr(lse), row0, _ptr(p), _ptr(ws), nb, _stream()))
    return o, lse, p


def debug_dkdv_tile_counts(counts):
    """counts: zeroed int64 CUDA tensor of 2 elements (tiles visited, tiles with non-zero P^F) or None; applies to
    attnqat_bwd calls on the current stream."""
    _check(lib().attnqat_debug_dkdv_tile_counts(_stream(), _ptr(counts) if counts is not None else None))


def debug_bwd_waves(waves: int):
    """Force the workgroup shape of the dQ and dK/dV passes (4 or 8 waves; 0 = automatic).  Process-wide."""
    _check(lib().attnqat_debug_bwd_waves(int(waves)))


def profile_enable(on: bool):
    """Per-kernel timing of the calls made on the current stream."""
    _check(lib().attnqat_profile_enable(_stream(), int(on)))


def profile_read():
    """[(kernel label, milliseconds)] of the most recent call on the current stream; synchronise the stream first."""
    ms = (ctypes.c_float * 16)()
    names = (ctypes.c_char_p * 16)()
    n = lib().attnqat_profile_read(_stream(), 16, ctypes.cast(ms, ctypes.c_void_p), ctypes.cast(names, ctypes.c_void_p))
    if n < 0:
        _check(n)
    return [(names[i].decode(), float(ms[i])) for i in range(n)]
