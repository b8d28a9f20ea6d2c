"""ctypes binding of libupipe.so (the C ABI in include/upipe.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  PyTorch supplies device memory and the current stream.  The
``upipe_*`` functions mirror the C entry points one to one; ``attn_fwd`` /
``attn_bwd`` / ``layer_fwd`` / ``layer_bwd`` are conveniences that allocate
outputs and the workspace with torch and raise on a non-zero status.

If the library has not been built this module raises when it is first used;
there is no fallback implementation.
"""

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libupipe.so")

UPIPE_OK = 0
STATUS = {0: "UPIPE_OK", -1: "UPIPE_ERR_INVALID_ARG", -2: "UPIPE_ERR_UNSUPPORTED",
          -3: "UPIPE_ERR_WORKSPACE", -4: "UPIPE_ERR_HIP"}

_c_void_p = ctypes.c_void_p
_i64 = ctypes.c_int64
_int = ctypes.c_int
_size = ctypes.c_size_t
_fptr = ctypes.c_void_p
_dbl = ctypes.c_double

class upipe_heads(ctypes.Structure):
    """Rows of heads in a larger tensor: pointer, row and head stride in elements."""
    _fields_ = [("p", _c_void_p), ("row", _i64), ("head", _i64)]


_SIGNATURES = {
    "upipe_status_string": (ctypes.c_char_p, [_int]),
    "upipe_version": (_int, []),
    "upipe_gqa_schedule": (_int, [_int, _int, _int, _int,
                                  ctypes.POINTER(_int), ctypes.POINTER(_int)]),
    "upipe_attn_fwd_workspace_size": (_size, [_i64, _int, _int, _int, _int]),
    "upipe_attn_bwd_workspace_size": (_size, [_i64, _int, _int, _int, _int]),
    "upipe_layer_fwd_workspace_size": (_size, [_i64, _int, _int, _int, _int, _int]),
    "upipe_layer_bwd_workspace_size": (_size, [_i64, _int, _int, _int, _int, _int]),
    "upipe_attn_fwd": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _fptr,
                              _i64, _int, _int, _int, _int, _int,
                              _c_void_p, _size, _c_void_p]),
    "upipe_attn_fwd_batch": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _fptr,
                                    _i64, _i64, _int, _int, _int, _int, _int,
                                    _c_void_p, _size, _c_void_p]),
    "upipe_attn_bwd": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _fptr,
                              _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                              _i64, _int, _int, _int, _int, _int,
                              _c_void_p, _size, _c_void_p]),
    "upipe_attn_bwd_batch": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _fptr,
                                    _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                                    _i64, _i64, _int, _int, _int, _int, _int,
                                    _c_void_p, _size, _c_void_p]),
    "upipe_attn_fwd_noalloc_scratch_bytes": (_size, []),
    "upipe_attn_fwd_noalloc": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _fptr,
                                      _i64, _int, _int, _int, _int, _int, _c_void_p]),
    "upipe_attn_fwd_ring_workspace_size": (_size, [_i64, _i64, _int, _int, _int, _int]),
    "upipe_attn_fwd_ring": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _fptr,
                                   _i64, _i64, _i64, _i64, _int, _int, _int, _int,
                                   _int, _c_void_p, _size, _c_void_p]),
    "upipe_lse_merge": (_int, [_c_void_p, _fptr, _c_void_p, _fptr, _i64, _int, _int,
                               _c_void_p]),
    "upipe_rope": (_int, [_c_void_p, _i64, _int, _int, _i64, _dbl, _int, _c_void_p]),
    "upipe_layer_fwd": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p,
                               _c_void_p, _fptr, _i64, _int, _int, _int, _int,
                               _int, _c_void_p, _size, _c_void_p]),
    "upipe_layer_bwd": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _fptr,
                               _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                               _i64, _int, _int, _int, _int, _int,
                               _c_void_p, _size, _c_void_p]),
    "upipe_layer_fwd_ex": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p,
                                  _c_void_p, _fptr, _i64, _i64, _int, _int, _int, _int,
                                  _int, _dbl, _i64, _c_void_p, _size, _c_void_p]),
    "upipe_layer_bwd_ex": (_int, [_c_void_p, _c_void_p, _c_void_p, _c_void_p, _fptr,
                                  _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                                  _i64, _i64, _int, _int, _int, _int, _int, _dbl, _i64,
                                  _c_void_p, _size, _c_void_p]),
    "upipe_gemm_bf16": (_int, [_c_void_p, _c_void_p, _c_void_p, _i64, _i64, _i64,
                               _c_void_p]),
    "upipe_varlen_plan_size": (_size, [_c_void_p, _c_void_p, _int, _int, _int, _int, _int]),
    "upipe_varlen_plan": (_int, [_c_void_p, _c_void_p, _int, _int, _int, _int, _int, _c_void_p,
                                 _size]),
    "upipe_attn_fwd_varlen_workspace_size": (_size, [_c_void_p]),
    "upipe_attn_fwd_varlen": (_int, [upipe_heads] * 4 + [_fptr, _i64, _c_void_p, _c_void_p,
                                                         _c_void_p, _size, _c_void_p]),
    "upipe_attn_bwd_varlen_workspace_size": (_size, [_c_void_p]),
    "upipe_attn_bwd_varlen": (_int, [upipe_heads] * 4 + [_fptr, _i64] + [upipe_heads] * 4 +
                              [_c_void_p, _c_void_p, _c_void_p, _size, _c_void_p]),
    "upipe_attn_decode_workspace_size": (_size, [_i64, _int, _i64, _i64, _int, _int, _int]),
    "upipe_attn_decode": (_int, [upipe_heads, upipe_heads, _i64, upipe_heads, _i64, _c_void_p,
                                 upipe_heads, upipe_heads, upipe_heads, _fptr, _i64, _int, _i64,
                                 _i64, _int, _int, _int, _c_void_p, _size, _c_void_p]),
    "upipe_qk_norm_rope": (_int, [upipe_heads, upipe_heads, _c_void_p, _c_void_p, _int,
                                  _c_void_p, upipe_heads, upipe_heads, _i64, _int, _int, _int,
                                  _dbl, _dbl, _c_void_p]),
    "upipe_qk_norm_rope_bwd_workspace_size": (_size, [_i64, _int, _int, _int]),
    "upipe_qk_norm_rope_bwd": (_int, [upipe_heads, upipe_heads, _c_void_p, _c_void_p, _int,
                                      _c_void_p] + [upipe_heads] * 4 +
                               [_c_void_p, _c_void_p, _i64, _int, _int, _int, _dbl, _dbl,
                                _c_void_p, _size, _c_void_p]),
    "upipe_profile_enable": (_int, [_int]),
    "upipe_profile_reset": (_int, []),
    "upipe_profile_query": (_int, [ctypes.c_char_p, ctypes.POINTER(_int),
                                   ctypes.POINTER(ctypes.c_double)]),
    "upipe_profile_name": (ctypes.c_char_p, [_int]),
}

_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with "
                "`python -m paper_2602_21196_amd.build` (no fallback exists)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


class UpipeError(RuntimeError):
    def __init__(self, fn, status):
        super().__init__(f"{fn} returned {STATUS.get(status, status)}")
        self.status = status


def _check(fn, status):
    if status != UPIPE_OK:
        raise UpipeError(fn, status)


# ------------------------------------------------------------ raw mirrors

def upipe_status_string(status):
    return lib().upipe_status_string(status).decode()


def upipe_version():
    return lib().upipe_version()


def upipe_gqa_schedule(H, Hkv, C, U):
    """Returns (status, stage_heads list[H], kv_stage list[Hkv])."""
    heads = (_int * max(H, 1))()
    kvs = (_int * max(Hkv, 1))()
    st = lib().upipe_gqa_schedule(H, Hkv, C, U, heads, kvs)
    return st, list(heads)[:H], list(kvs)[:Hkv]


def upipe_attn_fwd_workspace_size(S, Hq, Hkv, d, U):
    return lib().upipe_attn_fwd_workspace_size(S, Hq, Hkv, d, U)


def upipe_attn_bwd_workspace_size(S, Hq, Hkv, d, U):
    return lib().upipe_attn_bwd_workspace_size(S, Hq, Hkv, d, U)


def upipe_layer_fwd_workspace_size(S, d_model, Hq, Hkv, d, U):
    return lib().upipe_layer_fwd_workspace_size(S, d_model, Hq, Hkv, d, U)


def upipe_layer_bwd_workspace_size(S, d_model, Hq, Hkv, d, U):
    return lib().upipe_layer_bwd_workspace_size(S, d_model, Hq, Hkv, d, U)


def upipe_attn_fwd(q, k, v, o, lse, S, Hq, Hkv, d, causal, U, ws, ws_bytes, stream):
    return lib().upipe_attn_fwd(q, k, v, o, lse, S, Hq, Hkv, d, causal, U, ws,
                                ws_bytes, stream)


def upipe_attn_fwd_batch(q, k, v, o, lse, B, S, Hq, Hkv, d, causal, U, ws, ws_bytes,
                         stream):
    return lib().upipe_attn_fwd_batch(q, k, v, o, lse, B, S, Hq, Hkv, d, causal, U,
                                      ws, ws_bytes, stream)


def upipe_attn_bwd(q, k, v, o, lse, dout, dq, dk, dv, S, Hq, Hkv, d, causal,
                   U, ws, ws_bytes, stream):
    return lib().upipe_attn_bwd(q, k, v, o, lse, dout, dq, dk, dv, S, Hq, Hkv,
                                d, causal, U, ws, ws_bytes, stream)


def upipe_attn_bwd_batch(q, k, v, o, lse, dout, dq, dk, dv, B, S, Hq, Hkv, d,
                         causal, U, ws, ws_bytes, stream):
    return lib().upipe_attn_bwd_batch(q, k, v, o, lse, dout, dq, dk, dv, B, S, Hq,
                                      Hkv, d, causal, U, ws, ws_bytes, stream)


def upipe_attn_fwd_noalloc_scratch_bytes():
    return lib().upipe_attn_fwd_noalloc_scratch_bytes()


def upipe_attn_fwd_noalloc(q, k, v, o, lse, S, Hq, Hkv, d, causal, U, stream):
    return lib().upipe_attn_fwd_noalloc(q, k, v, o, lse, S, Hq, Hkv, d, causal, U, stream)


def upipe_attn_fwd_ring_workspace_size(Sq, Skv, Hq, Hkv, d, U):
    return lib().upipe_attn_fwd_ring_workspace_size(Sq, Skv, Hq, Hkv, d, U)


def upipe_attn_fwd_ring(q, k, v, o, lse, Sq, Skv, q_offset, kv_offset, Hq, Hkv,
                        d, causal, U, ws, ws_bytes, stream):
    return lib().upipe_attn_fwd_ring(q, k, v, o, lse, Sq, Skv, q_offset,
                                     kv_offset, Hq, Hkv, d, causal, U, ws,
                                     ws_bytes, stream)


def upipe_lse_merge(o, lse, o_part, lse_part, S, H, d, stream):
    return lib().upipe_lse_merge(o, lse, o_part, lse_part, S, H, d, stream)


def upipe_rope(x, S, H, d, pos0, base, inverse, stream):
    return lib().upipe_rope(x, S, H, d, pos0, base, inverse, stream)


def upipe_layer_fwd(x, wqkv, wo, y, o_saved, lse_saved, S, d_model, Hq, Hkv, d, U,
                    ws, ws_bytes, stream):
    return lib().upipe_layer_fwd(x, wqkv, wo, y, o_saved, lse_saved, S, d_model,
                                 Hq, Hkv, d, U, ws, ws_bytes, stream)


def upipe_layer_bwd(x, wqkv, wo, o_saved, lse_saved, dy, dx, dwqkv, dwo, S,
                    d_model, Hq, Hkv, d, U, ws, ws_bytes, stream):
    return lib().upipe_layer_bwd(x, wqkv, wo, o_saved, lse_saved, dy, dx,
                                 dwqkv, dwo, S, d_model, Hq, Hkv, d, U, ws,
                                 ws_bytes, stream)


def upipe_layer_fwd_ex(x, wqkv, wo, y, o_saved, lse_saved, B, S, d_model, Hq, Hkv,
                       d, U, rope_base, pos0, ws, ws_bytes, stream):
    return lib().upipe_layer_fwd_ex(x, wqkv, wo, y, o_saved, lse_saved, B, S,
                                    d_model, Hq, Hkv, d, U, rope_base, pos0, ws,
                                    ws_bytes, stream)


def upipe_layer_bwd_ex(x, wqkv, wo, o_saved, lse_saved, dy, dx, dwqkv, dwo, B, S,
                       d_model, Hq, Hkv, d, U, rope_base, pos0, ws, ws_bytes,
                       stream):
    return lib().upipe_layer_bwd_ex(x, wqkv, wo, o_saved, lse_saved, dy, dx,
                                    dwqkv, dwo, B, S, d_model, Hq, Hkv, d, U,
                                    rope_base, pos0, ws, ws_bytes, stream)


def upipe_gemm_bf16(a, b, c, M, N, K, stream):
    return lib().upipe_gemm_bf16(a, b, c, M, N, K, stream)


def upipe_varlen_plan_size(cu_q, cu_k, n_seq, Hq, Hkv, d, causal):
    return lib().upipe_varlen_plan_size(cu_q, cu_k, n_seq, Hq, Hkv, d, causal)


def upipe_varlen_plan(cu_q, cu_k, n_seq, Hq, Hkv, d, causal, plan, plan_bytes):
    return lib().upipe_varlen_plan(cu_q, cu_k, n_seq, Hq, Hkv, d, causal, plan, plan_bytes)


def upipe_attn_fwd_varlen_workspace_size(plan):
    return lib().upipe_attn_fwd_varlen_workspace_size(plan)


def upipe_attn_fwd_varlen(q, k, v, o, lse, lse_head, plan, plan_dev, ws, ws_bytes, stream):
    return lib().upipe_attn_fwd_varlen(q, k, v, o, lse, lse_head, plan, plan_dev, ws, ws_bytes,
                                       stream)


def upipe_attn_bwd_varlen_workspace_size(plan):
    return lib().upipe_attn_bwd_varlen_workspace_size(plan)


def upipe_attn_bwd_varlen(q, k, v, o, lse, lse_head, dout, dq, dk, dv, plan, plan_dev, ws, ws_bytes,
                          stream):
    return lib().upipe_attn_bwd_varlen(q, k, v, o, lse, lse_head, dout, dq, dk, dv, plan, plan_dev,
                                       ws, ws_bytes, stream)


def upipe_attn_decode_workspace_size(B, nq, cap, P, Hq, Hkv, d):
    return lib().upipe_attn_decode_workspace_size(B, nq, cap, P, Hq, Hkv, d)


def upipe_attn_decode(q, k, k_cache, v, v_cache, lens, k_prefix, v_prefix, o, lse, B, nq, cap, P,
                      Hq, Hkv, d, ws, ws_bytes, stream):
    return lib().upipe_attn_decode(q, k, k_cache, v, v_cache, lens, k_prefix, v_prefix, o, lse, B,
                                   nq, cap, P, Hq, Hkv, d, ws, ws_bytes, stream)


def upipe_qk_norm_rope(q, k, wq, wk, w_fp32, positions, q_out, k_out, T, Hq, Hkv, d, base, eps,
                       stream):
    return lib().upipe_qk_norm_rope(q, k, wq, wk, w_fp32, positions, q_out, k_out, T, Hq, Hkv, d,
                                    base, eps, stream)


def upipe_qk_norm_rope_bwd_workspace_size(T, Hq, Hkv, d):
    return lib().upipe_qk_norm_rope_bwd_workspace_size(T, Hq, Hkv, d)


def upipe_qk_norm_rope_bwd(q, k, wq, wk, w_fp32, positions, dq_out, dk_out, dq, dk, dwq, dwk, T,
                           Hq, Hkv, d, base, eps, ws, ws_bytes, stream):
    return lib().upipe_qk_norm_rope_bwd(q, k, wq, wk, w_fp32, positions, dq_out, dk_out, dq, dk,
                                        dwq, dwk, T, Hq, Hkv, d, base, eps, ws, ws_bytes, stream)


def upipe_profile_enable(on):
    return lib().upipe_profile_enable(int(on))


def upipe_profile_reset():
    return lib().upipe_profile_reset()


def upipe_profile_query(name):
    n = _int(0)
    ms = ctypes.c_double(0.0)
    st = lib().upipe_profile_query(name.encode(), ctypes.byref(n),
                                   ctypes.byref(ms))
    _check("upipe_profile_query", st)
    return n.value, ms.value


def upipe_profile_names():
    out, i = [], 0
    while True:
        nm = lib().upipe_profile_name(i)
        if nm is None:
            return out
        out.append(nm.decode())
        i += 1


# ------------------------------------------------------ torch conveniences

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _ptr(t, dtype, name):
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream():
    return _torch().cuda.current_stream().cuda_stream


def workspace(nbytes, device):
    torch = _torch()
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def _batch(t, rank):
    """(B, shape without the batch) of a tensor with an optional leading batch."""
    if t.dim() == rank:
        return 1, tuple(t.shape)
    if t.dim() == rank + 1:
        return t.shape[0], tuple(t.shape[1:])
    raise ValueError(f"expected {rank} or {rank + 1} dimensions, got {t.dim()}")


def _lse_shape(q, B, Hq, S):
    return (Hq, S) if q.dim() == 3 else (B, Hq, S)


def _shape(t, want, name):
    """Raise ValueError unless tensor t has exactly the shape `want`: the C ABI
    sees raw pointers only, so a wrong size would be read or written out of
    bounds on the GPU."""
    if tuple(t.shape) != tuple(want):
        raise ValueError(f"{name} must have shape {tuple(want)}, got {tuple(t.shape)}")


def _attn_shapes(q, k, v, lead):
    """(B, S, Hq, Hkv, d) of q [(B,)S,Hq,d], k and v [(B,)S,Hkv,d]."""
    if q.dim() not in (3, 4):
        raise ValueError(f"q must be [S,Hq,d] or [B,S,Hq,d], got {tuple(q.shape)}")
    B, (S, Hq, d) = _batch(q, 3)
    if k.dim() != q.dim():
        raise ValueError(f"k must have shape {lead}[S,Hkv,d] like q, got {tuple(k.shape)}")
    Hkv = k.shape[-2]
    _shape(k, tuple(q.shape[:-2]) + (Hkv, d), "k")
    _shape(v, tuple(q.shape[:-2]) + (Hkv, d), "v")
    return B, S, Hq, Hkv, d


def attn_fwd(q, k, v, causal=True, U=1, ws=None):
    """o [(B,)S,Hq,d] bf16, lse [(B,)Hq,S] fp32 for q [(B,)S,Hq,d],
    k/v [(B,)S,Hkv,d] bf16.  Without a batch dimension this is the contract
    call upipe_attn_fwd, with one upipe_attn_fwd_batch."""
    torch = _torch()
    B, S, Hq, Hkv, d = _attn_shapes(q, k, v, "[B,]")
    need = upipe_attn_fwd_workspace_size(S, Hq, Hkv, d, U)
    if need == 0:
        raise UpipeError("upipe_attn_fwd_workspace_size", -1)
    if ws is None:
        ws = workspace(need, q.device)
    o = torch.empty_like(q)
    lse = torch.empty(_lse_shape(q, B, Hq, S), dtype=torch.float32, device=q.device)
    bf = torch.bfloat16
    ptrs = (_ptr(q, bf, "q"), _ptr(k, bf, "k"), _ptr(v, bf, "v"), _ptr(o, bf, "o"),
            _ptr(lse, torch.float32, "lse"))
    if q.dim() == 3:
        st = upipe_attn_fwd(*ptrs, S, Hq, Hkv, d, int(causal), U, ws.data_ptr(),
                            ws.numel(), _stream())
        _check("upipe_attn_fwd", st)
    else:
        st = upipe_attn_fwd_batch(*ptrs, B, S, Hq, Hkv, d, int(causal), U, ws.data_ptr(),
                                  ws.numel(), _stream())
        _check("upipe_attn_fwd_batch", st)
    return o, lse


def attn_fwd_ring(q, k, v, q_offset, kv_offset, causal=True, U=1, ws=None):
    """One ring step: o [Sq,Hq,d] bf16, lse [Hq,Sq] fp32 of q [Sq,Hq,d] (global
    rows q_offset..) against k/v [Skv,Hkv,d] (global rows kv_offset..)."""
    torch = _torch()
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("attn_fwd_ring: q [Sq,Hq,d], k and v [Skv,Hkv,d]")
    Sq, Hq, d = q.shape
    Skv, Hkv = k.shape[0], k.shape[1]
    _shape(k, (Skv, Hkv, d), "k")
    _shape(v, (Skv, Hkv, d), "v")
    need = upipe_attn_fwd_ring_workspace_size(Sq, Skv, Hq, Hkv, d, U)
    if need == 0:
        raise UpipeError("upipe_attn_fwd_ring_workspace_size", -1)
    if ws is None:
        ws = workspace(need, q.device)
    o = torch.empty_like(q)
    lse = torch.empty((Hq, Sq), dtype=torch.float32, device=q.device)
    bf = torch.bfloat16
    st = upipe_attn_fwd_ring(_ptr(q, bf, "q"), _ptr(k, bf, "k"), _ptr(v, bf, "v"),
                             _ptr(o, bf, "o"), _ptr(lse, torch.float32, "lse"),
                             Sq, Skv, int(q_offset), int(kv_offset), Hq, Hkv, d,
                             int(causal), U, ws.data_ptr(), ws.numel(), _stream())
    _check("upipe_attn_fwd_ring", st)
    return o, lse


def lse_merge(o, lse, o_part, lse_part):
    """In place: fold (o_part [S,H,d], lse_part [H,S]) into (o, lse)."""
    torch = _torch()
    if o.dim() != 3:
        raise ValueError("lse_merge: o, o_part [S,H,d] and lse, lse_part [H,S]")
    S, H, d = o.shape
    if tuple(o_part.shape) != (S, H, d) or tuple(lse.shape) != (H, S) or \
            tuple(lse_part.shape) != (H, S):
        raise ValueError("lse_merge: o, o_part [S,H,d] and lse, lse_part [H,S]")
    bf = torch.bfloat16
    st = upipe_lse_merge(_ptr(o, bf, "o"), _ptr(lse, torch.float32, "lse"),
                         _ptr(o_part, bf, "o_part"),
                         _ptr(lse_part, torch.float32, "lse_part"), S, H, d, _stream())
    _check("upipe_lse_merge", st)
    return o, lse


def attn_bwd(q, k, v, o, lse, dout, causal=True, U=1, ws=None):
    """dq [(B,)S,Hq,d], dk, dv [(B,)S,Hkv,d] bf16.  Without a batch dimension
    this is the contract call upipe_attn_bwd, with one upipe_attn_bwd_batch."""
    torch = _torch()
    B, S, Hq, Hkv, d = _attn_shapes(q, k, v, "[B,]")
    _shape(o, q.shape, "o")
    _shape(dout, q.shape, "dout")
    _shape(lse, _lse_shape(q, B, Hq, S), "lse")
    need = upipe_attn_bwd_workspace_size(S, Hq, Hkv, d, U)
    if need == 0:
        raise UpipeError("upipe_attn_bwd_workspace_size", -1)
    if ws is None:
        ws = workspace(need, q.device)
    dq = torch.empty_like(q)
    dk = torch.empty_like(k)
    dv = torch.empty_like(v)
    bf = torch.bfloat16
    ptrs = (_ptr(q, bf, "q"), _ptr(k, bf, "k"), _ptr(v, bf, "v"), _ptr(o, bf, "o"),
            _ptr(lse, torch.float32, "lse"), _ptr(dout, bf, "dout"), _ptr(dq, bf, "dq"),
            _ptr(dk, bf, "dk"), _ptr(dv, bf, "dv"))
    if q.dim() == 3:
        st = upipe_attn_bwd(*ptrs, S, Hq, Hkv, d, int(causal), U, ws.data_ptr(),
                            ws.numel(), _stream())
        _check("upipe_attn_bwd", st)
    else:
        st = upipe_attn_bwd_batch(*ptrs, B, S, Hq, Hkv, d, int(causal), U, ws.data_ptr(),
                                  ws.numel(), _stream())
        _check("upipe_attn_bwd_batch", st)
    return dq, dk, dv


def rope(x, base, pos0=0, inverse=False):
    """In place on x [S,H,d] bf16: rotary embedding at positions pos0 + s."""
    torch = _torch()
    if x.dim() != 3:
        raise ValueError(f"rope: x must be [S,H,d], got {tuple(x.shape)}")
    S, H, d = x.shape
    st = upipe_rope(_ptr(x, torch.bfloat16, "x"), S, H, d, int(pos0), float(base),
                    int(bool(inverse)), _stream())
    _check("upipe_rope", st)
    return x


def _layer_shapes(x, wqkv, wo, Hq, Hkv, d):
    """(B, S, d_model) of x [(B,)S,dm], with wqkv and wo checked against the
    head counts."""
    if x.dim() not in (2, 3):
        raise ValueError(f"x must be [S,d_model] or [B,S,d_model], got {tuple(x.shape)}")
    B, (S, dm) = _batch(x, 2)
    _shape(wqkv, (dm, (Hq + 2 * Hkv) * d), "wqkv")
    _shape(wo, (Hq * d, dm), "wo")
    return B, S, dm


def _plain_layer(x, rope_base, pos0):
    """The contract calls cover one sequence without rotary embedding."""
    return x.dim() == 2 and float(rope_base) == 0.0 and int(pos0) == 0


def layer_fwd(x, wqkv, wo, Hq, Hkv, d=128, U=1, ws=None, rope_base=0.0, pos0=0):
    """y [(B,)S,dm] bf16, o_saved [(B,)S,Hq,d] bf16, lse_saved [(B,)Hq,S]
    fp32.  rope_base > 0 rotates Q and K at positions pos0 + s.  One sequence
    without rotation goes through the contract call upipe_layer_fwd, anything
    else through upipe_layer_fwd_ex."""
    torch = _torch()
    B, S, dm = _layer_shapes(x, wqkv, wo, Hq, Hkv, d)
    need = upipe_layer_fwd_workspace_size(S, dm, Hq, Hkv, d, U)
    if need == 0:
        raise UpipeError("upipe_layer_fwd_workspace_size", -1)
    if ws is None:
        ws = workspace(need, x.device)
    y = torch.empty_like(x)
    lead = (B,) if x.dim() == 3 else ()
    o = torch.empty(lead + (S, Hq, d), dtype=torch.bfloat16, device=x.device)
    lse = torch.empty(lead + (Hq, S), dtype=torch.float32, device=x.device)
    bf = torch.bfloat16
    ptrs = (_ptr(x, bf, "x"), _ptr(wqkv, bf, "wqkv"), _ptr(wo, bf, "wo"), _ptr(y, bf, "y"),
            _ptr(o, bf, "o_saved"), _ptr(lse, torch.float32, "lse_saved"))
    if _plain_layer(x, rope_base, pos0):
        st = upipe_layer_fwd(*ptrs, S, dm, Hq, Hkv, d, U, ws.data_ptr(), ws.numel(),
                             _stream())
        _check("upipe_layer_fwd", st)
    else:
        st = upipe_layer_fwd_ex(*ptrs, B, S, dm, Hq, Hkv, d, U, float(rope_base), int(pos0),
                                ws.data_ptr(), ws.numel(), _stream())
        _check("upipe_layer_fwd_ex", st)
    return y, o, lse


def layer_bwd(x, wqkv, wo, o_saved, lse_saved, dy, Hq, Hkv, d=128, U=1,
              ws=None, rope_base=0.0, pos0=0):
    """dx [(B,)S,dm], dwqkv [dm,(Hq+2Hkv)d], dwo [Hq d, dm] (summed over the
    batch), all bf16.  o_saved = lse_saved = None recomputes the attention
    output (full checkpointing) instead of reading the kept one.  One
    sequence without rotation goes through the contract call upipe_layer_bwd,
    anything else through upipe_layer_bwd_ex."""
    torch = _torch()
    B, S, dm = _layer_shapes(x, wqkv, wo, Hq, Hkv, d)
    _shape(dy, x.shape, "dy")
    kept = o_saved is not None
    if kept != (lse_saved is not None):
        raise ValueError("layer_bwd: pass both o_saved and lse_saved, or neither")
    lead = (B,) if x.dim() == 3 else ()
    if kept:
        _shape(o_saved, lead + (S, Hq, d), "o_saved")
        _shape(lse_saved, lead + (Hq, S), "lse_saved")
    need = upipe_layer_bwd_workspace_size(S, dm, Hq, Hkv, d, U)
    if need == 0:
        raise UpipeError("upipe_layer_bwd_workspace_size", -1)
    if ws is None:
        ws = workspace(need, x.device)
    dx = torch.empty_like(x)
    dwqkv = torch.empty_like(wqkv)
    dwo = torch.empty_like(wo)
    bf = torch.bfloat16
    ptrs = (_ptr(x, bf, "x"), _ptr(wqkv, bf, "wqkv"), _ptr(wo, bf, "wo"),
            _ptr(o_saved, bf, "o_saved") if kept else None,
            _ptr(lse_saved, torch.float32, "lse_saved") if kept else None,
            _ptr(dy, bf, "dy"), _ptr(dx, bf, "dx"), _ptr(dwqkv, bf, "dwqkv"),
            _ptr(dwo, bf, "dwo"))
    if _plain_layer(x, rope_base, pos0):
        st = upipe_layer_bwd(*ptrs, S, dm, Hq, Hkv, d, U, ws.data_ptr(), ws.numel(),
                             _stream())
        _check("upipe_layer_bwd", st)
    else:
        st = upipe_layer_bwd_ex(*ptrs, B, S, dm, Hq, Hkv, d, U, float(rope_base), int(pos0),
                                ws.data_ptr(), ws.numel(), _stream())
        _check("upipe_layer_bwd_ex", st)
    return dx, dwqkv, dwo


def gemm(a, b):
    """c [M,N] = a [M,K] . b [K,N], bf16 with fp32 accumulation (M, N, K
    multiples of 128)."""
    torch = _torch()
    if a.dim() != 2 or b.dim() != 2 or a.shape[1] != b.shape[0]:
        raise ValueError(f"gemm: a [M,K] and b [K,N], got {tuple(a.shape)}, {tuple(b.shape)}")
    M, K = a.shape
    N = b.shape[1]
    c = torch.empty((M, N), dtype=torch.bfloat16, device=a.device)
    bf = torch.bfloat16
    st = upipe_gemm_bf16(_ptr(a, bf, "a"), _ptr(b, bf, "b"), _ptr(c, bf, "c"), M, N, K,
                         _stream())
    _check("upipe_gemm_bf16", st)
    return c


# ------------------------------------------- rows in place: strides, devices

def _rows(t, name, shape=None):
    """upipe_heads of a bf16 GPU tensor [T, H, 128] whose rows of 128 are dense: a
    column block of a projection's output need not be copied."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name} must be {torch.bfloat16}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    size, stride = t.shape, t.stride()
    if len(size) != 3:
        raise ValueError(f"{name} must be [T,H,d], got {tuple(size)}")
    if shape is not None and size != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(size)}")
    T, H, d = size
    if d > 1 and stride[2] != 1:
        raise ValueError(f"{name} must have dense rows, got strides {stride}")
    head = stride[1] if H > 1 else d
    return upipe_heads(t.data_ptr(), stride[0] if T > 1 else H * head, head)


def _dense(t, shape, dtype, name):
    """Pointer of a dense GPU tensor of this shape (a tuple) and type."""
    if not isinstance(t, _torch().Tensor) or t.shape != shape or t.dtype is not dtype:
        _ptr(t, dtype, name)
        _shape(t, shape, name)
    if not (t.is_cuda and t.is_contiguous()):
        _ptr(t, dtype, name)
    return t.data_ptr()


def _new_rows(t):
    """A dense tensor like t [T, H, d] (new_empty(t.shape) takes half as long again), and
    its upipe_heads."""
    torch = _torch()
    new = torch.empty_like(t, memory_format=torch.contiguous_format)
    H, d = t.shape[-2:]
    return new, upipe_heads(new.data_ptr(), H * d, d)


def _call(fn, args, *tensors):
    """lib().fn(*args, stream) on the current stream of the tensors' device, made the
    current one; all of them (None: not given) have to be on it."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{fn}: tensors on different devices: " + ", ".join(
                str(t.device) for t in tensors if t is not None))
    torch = _torch()
    # the stream's handle; current_stream().cuda_stream makes an object of it first (2.5 us)
    stream = torch._C._cuda_getCurrentRawStream(dev)
    if torch.cuda.current_device() == dev:
        st = getattr(lib(), fn)(*args, stream)
    else:
        with torch.cuda.device(dev):
            st = getattr(lib(), fn)(*args, stream)
    if st != UPIPE_OK:
        raise UpipeError(fn, st)


def _workspace(ws, need, device, fn):
    """ws checked, or a new one of `need` bytes."""
    if need == 0:
        raise UpipeError(fn, -1)
    if ws is None:
        return workspace(need, device)
    _ptr(ws, _torch().uint8, "ws")
    return ws


# ----------------------------------------------- norm of heads with rotation

def _norm_inputs(q, k, wq, wk, positions):
    """(T, Hq, Hkv, views of q and k, pointers of weights and positions, fp32?)"""
    torch = _torch()
    vq = _rows(q, "q")
    T, Hq, d = q.shape
    vk = _rows(k, "k", (T, k.shape[1] if k.dim() == 3 else 1, d))
    w = wq.dtype
    if w is not torch.bfloat16 and w is not torch.float32:
        raise TypeError(f"wq must be bfloat16 or float32, got {w}")
    return (T, Hq, k.shape[1], vq, vk,
            (_dense(wq, (d,), w, "wq"), _dense(wk, (d,), w, "wk"), int(w is torch.float32),
             _dense(positions, (T,), torch.int64, "positions")))


def _pair_out(out, q, k, names):
    """The caller's two output tensors, like q and k, or two new dense ones, each with its
    upipe_heads."""
    if out is None:
        return *_new_rows(q), *_new_rows(k)
    a, b = out
    return a, _rows(a, names[0], q.shape), b, _rows(b, names[1], k.shape)


def qk_norm_rope(q, k, wq, wk, positions, base, eps=1e-6, out=None):
    """(q', k'): every head of q [T,Hq,d] and k [T,Hkv,d] normed over its d
    elements, times wq / wk [d] (bf16 or fp32), rotated at positions [T] (int64).
    q, k and out = (q', k') may be strided views with dense rows; out may be (q, k)."""
    T, Hq, Hkv, vq, vk, rest = _norm_inputs(q, k, wq, wk, positions)
    yq, vyq, yk, vyk = _pair_out(out, q, k, ("q_out", "k_out"))
    _call("upipe_qk_norm_rope",
          (vq, vk, *rest, vyq, vyk, T, Hq, Hkv, q.shape[2], float(base), float(eps)),
          q, k, wq, wk, positions, yq, yk)
    return yq, yk


def qk_norm_rope_bwd(q, k, wq, wk, positions, base, dq_out, dk_out, eps=1e-6, out=None, ws=None):
    """(dq, dk, dwq, dwk) from the inputs of qk_norm_rope and the gradients of its
    outputs.  out = (dq, dk) may be (dq_out, dk_out) or (q, k)."""
    torch = _torch()
    T, Hq, Hkv, vq, vk, rest = _norm_inputs(q, k, wq, wk, positions)
    vdy = _rows(dq_out, "dq_out", q.shape), _rows(dk_out, "dk_out", k.shape)
    dq, vdq, dk, vdk = _pair_out(out, q, k, ("dq", "dk"))
    dwq, dwk = torch.empty_like(wq), torch.empty_like(wk)
    ws = _workspace(ws, upipe_qk_norm_rope_bwd_workspace_size(T, Hq, Hkv, q.shape[2]), q.device,
                    "upipe_qk_norm_rope_bwd_workspace_size")
    _call("upipe_qk_norm_rope_bwd",
          (vq, vk, *rest, *vdy, vdq, vdk, dwq.data_ptr(), dwk.data_ptr(), T, Hq, Hkv, q.shape[2],
           float(base), float(eps), ws.data_ptr(), ws.numel()),
          q, k, wq, wk, positions, dq_out, dk_out, dq, dk, ws)
    return dq, dk, dwq, dwk


# --------------------------------------- packed sequences, caches, prefixes

def _offsets(cu, name):
    """A host list of offsets as a C array of int64."""
    torch = _torch()
    if isinstance(cu, torch.Tensor):
        if cu.is_cuda:
            raise ValueError(f"{name} is planned on the host: pass a list or a CPU tensor")
        cu = cu.tolist()
    cu = [int(x) for x in cu]
    if not cu:
        raise ValueError(f"{name} needs n + 1 offsets")
    return (_i64 * len(cu))(*cu), cu


class VarlenPlan:
    """The work of one batch of packed sequences: sequence s has the queries
    cu_q[s] .. cu_q[s+1] and the keys cu_k[s] .. cu_k[s+1] (the same, unless given).
    Host offsets, 0 first.  Made once per batch, for all layers, forward and backward, on
    any streams.  The kernels read its list on the device: keep the plan until the calls
    that were given it have run, and with a captured graph of such calls."""

    def __init__(self, cu_q, cu_k=None, *, Hq, Hkv, causal=True, device="cuda"):
        torch = _torch()
        c_q, cu_q = _offsets(cu_q, "cu_q")
        c_k, cu_k = (c_q, cu_q) if cu_k is None else _offsets(cu_k, "cu_k")
        if len(cu_q) != len(cu_k):
            raise ValueError(f"cu_q has {len(cu_q)} offsets, cu_k {len(cu_k)}")
        args = (c_q, c_k, len(cu_q) - 1, int(Hq), int(Hkv), 128, int(bool(causal)))
        need = upipe_varlen_plan_size(*args)
        if need == 0:
            raise UpipeError("upipe_varlen_plan_size", -1)
        self._host = bytearray(need)
        self._buf = (ctypes.c_char * need).from_buffer(self._host)
        self.host = ctypes.addressof(self._buf)
        _check("upipe_varlen_plan", upipe_varlen_plan(*args, self.host, need))
        self.Hq, self.Hkv, self.causal = int(Hq), int(Hkv), bool(causal)
        self.total_q, self.total_k = cu_q[-1], cu_k[-1]
        self.fwd_workspace = upipe_attn_fwd_varlen_workspace_size(self.host)
        self.bwd_workspace = upipe_attn_bwd_varlen_workspace_size(self.host)
        self.dev = torch.frombuffer(self._host, dtype=torch.uint8).to(device)


def _packed(t, name, rows, H):
    """upipe_heads of [>= rows, H, 128]."""
    v = _rows(t, name)
    if t.shape[0] < rows or t.shape[1] != H or t.shape[2] != 128:
        raise ValueError(f"{name} must be [T,{H},128] with T >= {rows}, got {tuple(t.shape)}")
    return v


def _packed_lse(lse, q, plan):
    T = q.shape[0]
    if lse.dim() != 2 or lse.shape[0] != plan.Hq or lse.shape[1] < T:
        raise ValueError(f"lse must be [{plan.Hq},{T}], got {tuple(lse.shape)}")
    return _ptr(lse, _torch().float32, "lse"), lse.shape[1]


def attn_fwd_varlen(q, k, v, plan, out=None, ws=None):
    """(o [T,Hq,d] bf16, lse [Hq,T] fp32) of the packed q [T,Hq,d], k, v [Tk,Hkv,d]
    (strided views with dense rows) of a VarlenPlan.  Rows behind the last sequence
    are left as they are in out = (o, lse), 0 and -inf in new tensors."""
    torch = _torch()
    Tq, Tk = plan.total_q, plan.total_k
    views = (_packed(q, "q", Tq, plan.Hq), _packed(k, "k", Tk, plan.Hkv),
             _packed(v, "v", Tk, plan.Hkv))
    if out is None:
        o, vo = _new_rows(q)
        lse = torch.empty(plan.Hq, q.shape[0], dtype=torch.float32, device=q.device)
        if Tq < q.shape[0]:
            o[Tq:] = 0
            lse[:, Tq:] = float("-inf")
    else:
        o, lse = out
        vo = _packed(o, "o", Tq, plan.Hq)
    ws = _workspace(ws, plan.fwd_workspace, q.device, "upipe_attn_fwd_varlen_workspace_size")
    _call("upipe_attn_fwd_varlen",
          (*views, vo, *_packed_lse(lse, q, plan), plan.host, plan.dev.data_ptr(), ws.data_ptr(),
           ws.numel()),
          q, k, v, o, lse, plan.dev, ws)
    return o, lse


def attn_bwd_varlen(q, k, v, o, lse, dout, plan, out=None, ws=None):
    """(dq, dk, dv) of the packed q, k, v, with o and lse of attn_fwd_varlen and the
    same plan.  Rows behind the last sequence are left as they are in out = (dq, dk, dv),
    0 in new tensors."""
    Tq, Tk = plan.total_q, plan.total_k
    views = (_packed(q, "q", Tq, plan.Hq), _packed(k, "k", Tk, plan.Hkv),
             _packed(v, "v", Tk, plan.Hkv), _packed(o, "o", Tq, plan.Hq))
    if out is None:
        (dq, vdq), (dk, vdk), (dv, vdv) = _new_rows(q), _new_rows(k), _new_rows(v)
        for t, n in ((dq, Tq), (dk, Tk), (dv, Tk)):
            if n < t.shape[0]:
                t[n:] = 0
    else:
        dq, dk, dv = out
        vdq, vdk, vdv = (_packed(dq, "dq", Tq, plan.Hq), _packed(dk, "dk", Tk, plan.Hkv),
                         _packed(dv, "dv", Tk, plan.Hkv))
    grads = (_packed(dout, "dout", Tq, plan.Hq), vdq, vdk, vdv)
    ws = _workspace(ws, plan.bwd_workspace, q.device, "upipe_attn_bwd_varlen_workspace_size")
    _call("upipe_attn_bwd_varlen",
          (*views, *_packed_lse(lse, q, plan), *grads, plan.host, plan.dev.data_ptr(),
           ws.data_ptr(), ws.numel()),
          q, k, v, o, lse, dout, dq, dk, dv, plan.dev, ws)
    return dq, dk, dv


def _cache(t, name, B, Hkv):
    """(upipe_heads of one cache, elements from one to the next) of [B, cap, Hkv, d]."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or t.dim() != 4:
        raise ValueError(f"{name} must be [B,cap,Hkv,d]")
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name} must be {torch.bfloat16}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    cap = t.shape[1]
    if t.shape != (B, cap, Hkv, 128):
        _shape(t, (B, cap, Hkv, 128), name)
    step, row, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{name} must have dense rows, got strides {t.stride()}")
    head = head if Hkv > 1 else 128
    return upipe_heads(t.data_ptr(), row if cap > 1 else Hkv * head, head), step if B > 1 else 0


def attn_decode(q, k_cache, v_cache, lens, k_prefix=None, v_prefix=None, out=None, ws=None):
    """(o like q, lse [B,Hq,nq] fp32) of the new tokens q [B,nq,Hq,d] against the caches
    [B,cap,Hkv,d], of which lens [B] (int32, on the device) rows are valid, the new tokens'
    own among them, behind the rows [P,Hkv,d] of a prefix that all share, if given."""
    torch = _torch()
    if q.dim() != 4:
        raise ValueError(f"q must be [B,nq,Hq,d], got {tuple(q.shape)}")
    if k_cache.dim() != 4 or k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache must be [B,cap,Hkv,d], got "
                         f"{tuple(k_cache.shape)}, {tuple(v_cache.shape)}")
    if (k_prefix is None) != (v_prefix is None):
        raise ValueError("attn_decode: pass both k_prefix and v_prefix, or neither")
    B, nq, Hq, d = q.shape
    cap, Hkv = k_cache.shape[1:3]
    if B < 1 or cap < 1:
        raise ValueError(f"attn_decode: no sequences or no cache rows ({B}, {cap})")
    if lens.shape != (B,):
        _shape(lens, (B,), "lens")
    vq = _rows(_flat_tokens(q, "q"), "q")
    vk, k_step = _cache(k_cache, "k_cache", B, Hkv)
    vv, v_step = _cache(v_cache, "v_cache", B, Hkv)
    P, none = 0, upipe_heads(None, 0, 0)
    vkp = vvp = none
    if k_prefix is not None:
        P = k_prefix.shape[0]
        vkp = _rows(k_prefix, "k_prefix", (P, Hkv, d))
        vvp = _rows(v_prefix, "v_prefix", (P, Hkv, d))
    if out is None:
        o, vo = _new_rows(q)
        lse = torch.empty(B, Hq, nq, dtype=torch.float32, device=q.device)
    else:
        o, lse = out
        _shape(o, q.shape, "o")
        vo = _rows(_flat_tokens(o, "o"), "o")
    need = upipe_attn_decode_workspace_size(B, nq, cap, P, Hq, Hkv, d)
    ws = _workspace(ws, need, q.device, "upipe_attn_decode_workspace_size")
    _call("upipe_attn_decode",
          (vq, vk, k_step, vv, v_step, _dense(lens, (B,), torch.int32, "lens"), vkp,
           vvp, vo, _dense(lse, (B, Hq, nq), torch.float32, "lse"), B, nq, cap, P, Hq,
           Hkv, d, ws.data_ptr(), ws.numel()),
          q, k_cache, v_cache, lens, k_prefix, v_prefix, o, lse, ws)
    return o, lse


def _flat_tokens(t, name):
    """[B, nq, H, d] as [B nq, H, d], without a copy."""
    try:
        return t.view(t.shape[0] * t.shape[1], *t.shape[2:])
    except RuntimeError:
        raise ValueError(f"{name}: the tokens of all sequences must be evenly spaced, got "
                         f"strides {t.stride()}") from None
