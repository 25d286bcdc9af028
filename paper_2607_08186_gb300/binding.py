"""Thin ctypes binding over libhdsfa.so (C ABI in include/hdsfa.h).

Argument marshalling only: every step of the computation runs in the CUDA
kernels of libhdsfa.so.  Functions keep the C names and take torch CUDA tensors
(plain device memory); sizes are read from the tensor shapes.  There is no
CPU fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

from .inputs import WITHIN, CROSS, LOCAL  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhdsfa.so")
_lock = threading.Lock()
_lib = None

HD_OK = 0
HD_DEVBIT_INDEX = 1
HD_DEVBIT_TIMEOUT = 2
HD_DEVBIT_PAGES = 4


class HdError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {hd_status_string(code)} (code {code})")
        self.code = code


def lib():
    """Load libhdsfa.so (built by ``build.build()``); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"libhdsfa.so is not built ({LIB_PATH}); run "
                                   "paper_2607_08186_gb300.build.build() first")
            L = ctypes.CDLL(LIB_PATH)
            P, I, F, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
            L.hd_selftest_bounded_wait.restype = I
            L.hd_selftest_bounded_wait.argtypes = [P, P, P]
            L.hd_expand_embed.restype = I
            L.hd_expand_embed.argtypes = [P, P, P, I, I, I, I, I, P, P]
            L.hd_expand_embed_bwd_workspace_bytes.restype = Z
            L.hd_expand_embed_bwd_workspace_bytes.argtypes = [I, I]
            L.hd_expand_embed_bwd.restype = I
            L.hd_expand_embed_bwd.argtypes = [P, P, P, I, I, I, I, I, P, Z, P, P]
            L.hd_expand_embed_bwd_plan.restype = I
            L.hd_expand_embed_bwd_plan.argtypes = [P, I, I, I, P, Z, P, P]
            L.hd_expand_embed_bwd_apply.restype = I
            L.hd_expand_embed_bwd_apply.argtypes = [P, P, I, I, I, I, I, P, Z, P]
            L.hd_select_final_stream.restype = I
            L.hd_select_final_stream.argtypes = [P, P, I, I, I, I, P]
            L.hd_select_final_stream_bwd.restype = I
            L.hd_select_final_stream_bwd.argtypes = [P, P, I, I, I, I, P]
            L.sfa_fwd_final.restype = I
            L.sfa_fwd_final.argtypes = [P, P, P, P, P, I, I, I, I, I, I, F, I, I, P, P]
            L.sfa_bwd_final_workspace_bytes.restype = Z
            L.sfa_bwd_final_workspace_bytes.argtypes = [I, I, I, I, I, I, I]
            L.sfa_bwd_final.restype = I
            L.sfa_bwd_final.argtypes = [P, P, P, P, P, P, P, P, P, I, I, I, I, I, I, F, I, I, P, Z, P, P]
            L.sfa_decode_workspace_bytes.restype = Z
            L.sfa_decode_workspace_bytes.argtypes = [I, I, I, I, I, I, I, I]
            L.sfa_decode.restype = I
            L.sfa_decode.argtypes = [P, P, P, P, P, P, I, I, I, I, I, I, I, F, I, I, P, Z, P, P]
            L.sfa_kv_append.restype = I
            L.sfa_kv_append.argtypes = [P, P, P, P, P, I, I, I, I, I, P, P]
            L.sfa_fwd_packed_workspace_bytes.restype = Z
            L.sfa_fwd_packed_workspace_bytes.argtypes = [I, I, I, I, I, I, I]
            L.sfa_fwd_packed.restype = I
            L.sfa_fwd_packed.argtypes = [P, P, P, P, P, P, I, I, I, I, I, I, F, I, I, P, Z, P, P]
            L.sfa_decode_paged_workspace_bytes.restype = Z
            L.sfa_decode_paged_workspace_bytes.argtypes = [I, I, I, I, I, I, I, I]
            L.sfa_decode_paged.restype = I
            L.sfa_decode_paged.argtypes = [P, P, P, P, P, P, P, I, I, I, I, I, I, I, I, I, F, I, I, P, Z, P, P]
            L.sfa_kv_append_paged.restype = I
            L.sfa_kv_append_paged.argtypes = [P, P, P, P, P, P, P, I, I, I, I, I, I, I, I, P, P]
            L.sfa_kv_append_paged_served.restype = I
            L.sfa_kv_append_paged_served.argtypes = [P, P, P, P, P, P, P, P, I, I, I, I, I, I, I, I, P, P]
            L.hd_pages_workspace_bytes.restype = Z
            L.hd_pages_workspace_bytes.argtypes = [I, I]
            L.hd_pages_grow.restype = I
            L.hd_pages_grow.argtypes = [P, P, P, P, I, I, I, I, P, Z, P, P]
            L.hd_pages_grow_served.restype = I
            L.hd_pages_grow_served.argtypes = [P, P, P, P, P, I, I, I, I, P, Z, P, P]
            L.hd_pages_fork.restype = I
            L.hd_pages_fork.argtypes = [P, P, P, P, P, P, I, P, I, I, I, I, P, Z, P, P]
            L.hd_pages_free.restype = I
            L.hd_pages_free.argtypes = [P, P, P, P, I, I, I, I, I, P, P]
            L.hd_pages_compact.restype = I
            L.hd_pages_compact.argtypes = [P, P, P, P, P, P, I, I, I, I, P, Z, P, P]
            L.hd_pages_copy.restype = I
            L.hd_pages_copy.argtypes = [P, P, P, I, I, Z, P, P]
            L.sfa_kv_append_paged_q8.restype = I
            L.sfa_kv_append_paged_q8.argtypes = [P] * 10 + [I] * 9 + [P, P]
            L.sfa_kv_read_paged_q8.restype = I
            L.sfa_kv_read_paged_q8.argtypes = [P] * 9 + [I] * 9 + [P, P]
            L.sfa_decode_paged_q8_workspace_bytes.restype = Z
            L.sfa_decode_paged_q8_workspace_bytes.argtypes = [I] * 8
            L.sfa_decode_paged_q8.restype = I
            L.sfa_decode_paged_q8.argtypes = [P] * 9 + [I] * 10 + [F, I, I, P, Z, P, P]
            L.hd_pages_copy_q8.restype = I
            L.hd_pages_copy_q8.argtypes = [P] * 5 + [I, I, Z, Z, P, P]
            L.sfa_fwd.restype = I
            L.sfa_fwd.argtypes = [P, P, P, P, P, I, I, I, I, I, I, F, I, I, P, P]
            L.sfa_bwd_workspace_bytes.restype = Z
            L.sfa_bwd_workspace_bytes.argtypes = [I, I, I, I, I, I, I]
            L.sfa_bwd.restype = I
            L.sfa_bwd.argtypes = [P, P, P, P, P, P, P, P, P, I, I, I, I, I, I, F, I, I, P, Z, P, P]
            L.sfa_bwd_prep.restype = I
            L.sfa_bwd_prep.argtypes = [P, P, P, I, I, I, I, I, I, I, P, Z, P]
            L.sfa_bwd_row_terms.restype = I
            L.sfa_bwd_row_terms.argtypes = [P, P, P, I, I, I, I, I, I, I, P, Z, P]
            L.sfa_bwd_clear.restype = I
            L.sfa_bwd_clear.argtypes = [I, I, I, I, I, I, I, P, Z, P]
            L.sfa_bwd_main.restype = I
            L.sfa_bwd_main.argtypes = [P, P, P, P, P, P, I, I, I, I, I, I, F, I, I, P, Z, P, P]
            L.sfa_bwd_finalize.restype = I
            L.sfa_bwd_finalize.argtypes = [P, I, I, I, I, I, I, F, I, P, Z, P]
            L.sfa_bwd_noalloc.restype = I
            L.sfa_bwd_noalloc.argtypes = [P, P, P, P, P, P, P, P, P, I, I, I, I, I, I, F, I, I, P, P]
            L.hd_status_string.restype = ctypes.c_char_p
            L.hd_status_string.argtypes = [I]
            _lib = L
    return _lib


def hd_status_string(code: int) -> str:
    return lib().hd_status_string(int(code)).decode()


def hd_selftest_bounded_wait(dev_status, dev_result, stream=None):
    """Diagnostic: one warp's bounded wait on a barrier nothing arrives on runs out
    (about a second); HD_DEVBIT_TIMEOUT lands in dev_status, 0 in dev_result."""
    _check(lib().hd_selftest_bounded_wait(_p(dev_status), _p(dev_result), _stream(stream)),
           "hd_selftest_bounded_wait")


def _p(t):
    """Device address of a tensor: a plain int, which the declared argument types convert."""
    return None if t is None else t.data_ptr()


# The current stream's handle without building a Stream object: that took 3 us of the 6 us
# a call spent outside the library (a short layer's or decoding step's calls are bound by
# their host time: a tiny forward + backward, with the padding kernel gone, 27.7 -> 18.5 us, append + decode at 100 tokens
# 22.1 -> 13.7, the four embedding calls at 128 tokens 37.2 -> 28.7).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(torch.cuda.current_device())
    return stream.cuda_stream


def _check(code: int, where: str):
    if code != HD_OK:
        raise HdError(code, where)


def hd_expand_embed(tables, ids, out, dev_status=None, stream=None):
    """out[b][t*n+s] = tables[s][ids[b][t]]  (Eq. 1).  tables [n][V][D] bf16,
    ids [B][L] int32, out [B][n*L][D] bf16."""
    n, V, D = tables.shape
    B, L = ids.shape
    _check(lib().hd_expand_embed(_p(tables), _p(ids), _p(out), B, L, n, V, D, _p(dev_status),
                                 _stream(stream)), "hd_expand_embed")
    return out


def hd_expand_embed_bwd_workspace_bytes(B, L) -> int:
    return int(lib().hd_expand_embed_bwd_workspace_bytes(B, L))


def hd_expand_embed_bwd(dout, ids, dtables, workspace, dev_status=None, stream=None):
    """dtables[s][v] += sum of dout[b][t*n+s] over tokens with ids[b][t] = v (adjoint of Eq. 1).
    dout [B][n*L][D] bf16, ids [B][L] int32, dtables [n][V][D] float32 (accumulated in place),
    workspace: uint8 CUDA tensor of >= hd_expand_embed_bwd_workspace_bytes(B, L) bytes."""
    n, V, D = dtables.shape
    B, L = ids.shape
    if dout.shape[1] != n * L:
        raise ValueError("dout.shape[1] must be n * L")
    _check(lib().hd_expand_embed_bwd(_p(dout), _p(ids), _p(dtables), B, L, n, V, D, _p(workspace),
                                     _wsb(workspace), _p(dev_status), _stream(stream)),
           "hd_expand_embed_bwd")
    return dtables


def hd_expand_embed_bwd_plan(ids, V, workspace, dev_status=None, stream=None):
    """The id-only part of hd_expand_embed_bwd: tokens sorted by id and each id's run,
    written into workspace for later hd_expand_embed_bwd_apply calls."""
    B, L = ids.shape
    _check(lib().hd_expand_embed_bwd_plan(_p(ids), B, L, int(V), _p(workspace), _wsb(workspace),
                                          _p(dev_status), _stream(stream)), "hd_expand_embed_bwd_plan")


def hd_expand_embed_bwd_apply(dout, dtables, workspace, L, stream=None):
    """dtables += the expansion backward of dout following the plan held in workspace
    (built by hd_expand_embed_bwd_plan for the same ids, B = dout.shape[0], L and V)."""
    n, V, D = dtables.shape
    B = dout.shape[0]
    if dout.shape[1] != n * L:
        raise ValueError("dout.shape[1] must be n * L")
    _check(lib().hd_expand_embed_bwd_apply(_p(dout), _p(dtables), B, L, n, V, D, _p(workspace),
                                           _wsb(workspace), _stream(stream)), "hd_expand_embed_bwd_apply")
    return dtables


def hd_select_final_stream(x, y, n, stream=None):
    """y[b][t] = x[b][t*n + n-1], the rows the loss reads (Eq. 2).  x [B][n*L][D], y [B][L][D] bf16."""
    B, L, D = y.shape
    if x.shape[1] != n * L:
        raise ValueError("x.shape[1] must be n * L")
    _check(lib().hd_select_final_stream(_p(x), _p(y), B, L, n, D, _stream(stream)),
           "hd_select_final_stream")
    return y


def hd_select_final_stream_bwd(dy, dx, n, stream=None):
    """dx[b][t*n + n-1] = dy[b][t], zero elsewhere.  dy [B][L][D], dx [B][n*L][D] bf16."""
    B, L, D = dy.shape
    if dx.shape[1] != n * L:
        raise ValueError("dx.shape[1] must be n * L")
    _check(lib().hd_select_final_stream_bwd(_p(dy), _p(dx), B, L, n, D, _stream(stream)),
           "hd_select_final_stream_bwd")
    return dx


def _attn_dims(q, k, n):
    B, nL, Hq, Dh = q.shape
    if nL % n:
        raise ValueError("q.shape[1] must be n * L")
    return B, nL // n, Hq, k.shape[2], Dh


def sfa_fwd(q, k, v, o, lse, n, mode, softmax_scale=0.0, window=0, dev_status=None, stream=None):
    """SFA forward (Eq. 4 / Fig. 2 masks).  q,o [B][nL][Hq][Dh], k,v [B][nL][Hkv][Dh] bf16;
    lse [B][Hq][nL] float32."""
    B, L, Hq, Hkv, Dh = _attn_dims(q, k, n)
    _check(lib().sfa_fwd(_p(q), _p(k), _p(v), _p(o), _p(lse), B, L, n, Hq, Hkv, Dh,
                         float(softmax_scale), int(mode), int(window), _p(dev_status),
                         _stream(stream)), "sfa_fwd")
    return o, lse


def sfa_bwd_workspace_bytes(B, L, n, Hq, Hkv, Dh, mode) -> int:
    return int(lib().sfa_bwd_workspace_bytes(B, L, n, Hq, Hkv, Dh, int(mode)))


def sfa_bwd(q, k, v, o, lse, dout, dq, dk, dv, n, mode, workspace, softmax_scale=0.0, window=0,
            dev_status=None, stream=None):
    """SFA backward.  workspace: uint8 CUDA tensor of >= sfa_bwd_workspace_bytes bytes."""
    B, L, Hq, Hkv, Dh = _attn_dims(q, k, n)
    _check(lib().sfa_bwd(_p(q), _p(k), _p(v), _p(o), _p(lse), _p(dout), _p(dq), _p(dk), _p(dv),
                         B, L, n, Hq, Hkv, Dh, float(softmax_scale), int(mode), int(window),
                         _p(workspace), _wsb(workspace),
                         _p(dev_status), _stream(stream)), "sfa_bwd")
    return dq, dk, dv


def _final_dims(q, k):
    B, L, Hq, Dh = q.shape
    if k.shape[1] % L:
        raise ValueError("k.shape[1] must be n * L")
    return B, L, k.shape[1] // L, Hq, k.shape[2], Dh


def sfa_fwd_final(q, k, v, o, lse, mode, softmax_scale=0.0, window=0, dev_status=None, stream=None):
    """Final-stream queries only (Eq. 2 rows; Sec. 3.1 final-stream-only layers): q, o [B][L][Hq][Dh],
    k, v [B][n*L][Hkv][Dh] bf16, lse [B][Hq][L] float32."""
    B, L, n, Hq, Hkv, Dh = _final_dims(q, k)
    _check(lib().sfa_fwd_final(_p(q), _p(k), _p(v), _p(o), _p(lse), B, L, n, Hq, Hkv, Dh, float(softmax_scale),
                               int(mode), int(window), _p(dev_status), _stream(stream)), "sfa_fwd_final")
    return o, lse


def sfa_bwd_final_workspace_bytes(B, L, n, Hq, Hkv, Dh, mode) -> int:
    return int(lib().sfa_bwd_final_workspace_bytes(B, L, n, Hq, Hkv, Dh, int(mode)))


def sfa_bwd_final(q, k, v, o, lse, dout, dq, dk, dv, mode, workspace, softmax_scale=0.0, window=0,
                  dev_status=None, stream=None):
    """Backward of sfa_fwd_final: dq [B][L][Hq][Dh], dk, dv [B][n*L][Hkv][Dh] (overwritten)."""
    B, L, n, Hq, Hkv, Dh = _final_dims(q, k)
    _check(lib().sfa_bwd_final(_p(q), _p(k), _p(v), _p(o), _p(lse), _p(dout), _p(dq), _p(dk), _p(dv), B, L, n, Hq,
                               Hkv, Dh, float(softmax_scale), int(mode), int(window), _p(workspace),
                               _wsb(workspace), _p(dev_status), _stream(stream)), "sfa_bwd_final")
    return dq, dk, dv


def sfa_decode_workspace_bytes(B, max_tokens, n, Hq, Hkv, Dh, mode, window=0) -> int:
    return int(lib().sfa_decode_workspace_bytes(B, max_tokens, n, Hq, Hkv, Dh, int(mode), int(window)))


def sfa_decode(q, k_cache, v_cache, lens, o, n, mode, workspace, max_tokens=None, lse=None, softmax_scale=0.0,
               window=0, dev_status=None, stream=None):
    """One decoding step (Sec. 3.2): the new token's n positions q [B][n][Hq][Dh] against
    the cache k_cache / v_cache [B][Lcap*n][Hkv][Dh] holding lens[b] tokens (int32 CUDA
    tensor [B]); o [B][n][Hq][Dh] bf16, lse [B][Hq][n] float32 or None.  max_tokens bounds
    every lens[b] (default: the cache capacity Lcap)."""
    B, nq, Hq, Dh = q.shape
    if nq != n or k_cache.shape[1] % n:
        raise ValueError("q.shape[1] must be n and k_cache.shape[1] a multiple of n")
    Lcap, Hkv = k_cache.shape[1] // n, k_cache.shape[2]
    T = Lcap if max_tokens is None else int(max_tokens)
    _check(lib().sfa_decode(_p(q), _p(k_cache), _p(v_cache), _p(lens), _p(o), _p(lse), B, T, Lcap, n, Hq, Hkv,
                            Dh, float(softmax_scale), int(mode), int(window), _p(workspace), _wsb(workspace),
                            _p(dev_status), _stream(stream)), "sfa_decode")
    return o


def sfa_kv_append(k_new, v_new, k_cache, v_cache, lens, n, dev_status=None, stream=None):
    """k_cache[b][(lens[b]-1)*n + s] = k_new[b][s] (and v): the new token's n K/V rows."""
    B, nn, Hkv, Dh = k_new.shape
    if nn != n:
        raise ValueError("k_new.shape[1] must be n")
    Lcap = k_cache.shape[1] // n
    _check(lib().sfa_kv_append(_p(k_new), _p(v_new), _p(k_cache), _p(v_cache), _p(lens), B, Lcap, n, Hkv, Dh,
                               _p(dev_status), _stream(stream)), "sfa_kv_append")


# ---- paged cache, pages and packed prompts.  These calls check their tensors: a wrong type,
# shape, layout or device raises ValueError before anything is enqueued.

def _tensors(stream, *args):
    """Check each of args, (name, tensor, dtype, shape) or None for what the caller left out; the stream's handle.
    (A call's host time is what a short step takes: the checks are about 0.4 us a tensor.)"""
    dev = args[0][1].get_device()  # -1: not on a CUDA device
    for a in args:
        if a is not None:
            name, t, dtype, shape = a
            if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
                _refuse(dev, name, t, dtype, shape)
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{args[0][0]} is on {args[0][1].device}; it must be on the current CUDA device")
    if stream is None:
        return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream
    if stream.device_index != dev:
        raise ValueError("stream belongs to another device than the current one")
    return stream.cuda_stream


def _refuse(dev, name, t, dtype, shape):
    if t.dtype is dtype and t.shape == shape and t.is_contiguous():
        raise ValueError(f"{name} is on {t.device}; all tensors must be on the current CUDA device")
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}, not {t.dtype} "
                     f"{tuple(t.shape)}{'' if t.is_contiguous() else ' (not contiguous)'}")


_BF16, _F32, _I32, _F8 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn


def _opt(name, t, dtype, shape):
    return None if t is None else (name, t, dtype, shape)


def _workspace(ws):
    if ws is None:
        raise ValueError("workspace must be a uint8 CUDA tensor")
    return "workspace", ws, torch.uint8, (ws.numel(),)


def _dev_status(st):
    return None if st is None else ("dev_status", st, _I32, (1,))


def sfa_fwd_packed_workspace_bytes(B, N, n, Hq, Hkv, Dh, mode) -> int:
    return int(lib().sfa_fwd_packed_workspace_bytes(B, N, n, Hq, Hkv, Dh, int(mode)))


def sfa_fwd_packed(q, k, v, o, lse, offsets, n, mode, workspace, softmax_scale=0.0, window=0, dev_status=None,
                   stream=None):
    """sfa_fwd over whole prompts of different lengths, packed: q, o [N*n][Hq][Dh], k, v [N*n][Hkv][Dh] bf16, lse
    [Hq][N*n] float32; sequence b holds tokens offsets[b] .. offsets[b+1]-1 (int32 [B+1], ascending, within [0, N]).
    Rows outside [offsets[0], offsets[B]) are left as they were."""
    if q.dim() != 3 or k.dim() != 3 or offsets.dim() != 1:
        raise ValueError("q must be [N*n][Hq][Dh], k [N*n][Hkv][Dh] and offsets [B+1]")
    rows, Hq, Dh = q.shape
    Hkv, B = k.shape[1], offsets.shape[0] - 1
    if n < 1 or rows % n:
        raise ValueError("q.shape[0] must be N * n")
    st = _tensors(stream, ("q", q, _BF16, (rows, Hq, Dh)), ("k", k, _BF16, (rows, Hkv, Dh)),
                  ("v", v, _BF16, (rows, Hkv, Dh)), ("o", o, _BF16, (rows, Hq, Dh)), ("lse", lse, _F32, (Hq, rows)),
                  ("offsets", offsets, _I32, (B + 1,)),
                  _workspace(workspace), _dev_status(dev_status))
    _check(lib().sfa_fwd_packed(_p(q), _p(k), _p(v), _p(o), _p(lse), _p(offsets), B, rows // n, n, Hq, Hkv, Dh,
                                float(softmax_scale), int(mode), int(window), _p(workspace), workspace.numel(),
                                _p(dev_status), st), "sfa_fwd_packed")
    return o, lse


def _pool_dims(k_pages, page_table, n):
    """(num_pages, page_tokens, Hkv, Dh, B, max_pages) of a paged cache."""
    if k_pages.dim() != 4 or page_table.dim() != 2:
        raise ValueError("k_pages must be [num_pages][page_tokens*n][Hkv][Dh] and page_table [B][max_pages]")
    pages, rows, Hkv, Dh = k_pages.shape
    if n < 1 or rows % n:
        raise ValueError("k_pages.shape[1] must be page_tokens * n")
    return pages, rows // n, Hkv, Dh, *page_table.shape


def sfa_kv_append_paged(k_new, v_new, k_pages, v_pages, page_table, lens, n, offsets=None, dev_status=None,
                        stream=None, served=None):
    """New tokens' K/V rows into a paged cache: pools [num_pages][page_tokens*n][Hkv][Dh] bf16, page_table
    [B][max_pages] and lens [B] int32 (the new tokens counted).  Without offsets k_new, v_new [B][n][Hkv][Dh] hold one
    token a sequence (a slot with lens 0 is left out); with offsets [B+1] int32, packed rows [N*n][Hkv][Dh], tokens
    offsets[b] .. offsets[b+1]-1 are the last ones of sequence b.  served [B] int32 (hd_pages_grow's): a sequence that
    got fewer tokens than it brings is left out."""
    pages, P, Hkv, Dh, B, width = _pool_dims(k_pages, page_table, n)
    if offsets is None:
        N, shape = B, (B, n, Hkv, Dh)
    else:
        N = k_new.shape[0] // n if k_new.dim() == 3 else 0
        shape = (N * n, Hkv, Dh)
    st = _tensors(stream, ("k_new", k_new, _BF16, shape), ("v_new", v_new, _BF16, shape),
                  ("k_pages", k_pages, _BF16, k_pages.shape), ("v_pages", v_pages, _BF16, k_pages.shape),
                  ("page_table", page_table, _I32, (B, width)), ("lens", lens, _I32, (B,)),
                  _opt("offsets", offsets, _I32, (B + 1,)), _opt("served", served, _I32, (B,)), _dev_status(dev_status))
    if served is not None:
        _check(lib().sfa_kv_append_paged_served(_p(k_new), _p(v_new), _p(k_pages), _p(v_pages), _p(page_table), _p(lens),
                                                _p(offsets), _p(served), B, N, pages, P, width, n, Hkv, Dh,
                                                _p(dev_status), st), "sfa_kv_append_paged_served")
        return
    _check(lib().sfa_kv_append_paged(_p(k_new), _p(v_new), _p(k_pages), _p(v_pages), _p(page_table), _p(lens),
                                     _p(offsets), B, N, pages, P, width, n, Hkv, Dh, _p(dev_status), st),
           "sfa_kv_append_paged")


def sfa_decode_paged_workspace_bytes(B, max_tokens, n, Hq, Hkv, Dh, mode, window=0) -> int:
    return int(lib().sfa_decode_paged_workspace_bytes(B, max_tokens, n, Hq, Hkv, Dh, int(mode), int(window)))


def sfa_decode_paged(q, k_pages, v_pages, page_table, lens, o, n, mode, workspace, max_tokens=None, lse=None,
                     softmax_scale=0.0, window=0, dev_status=None, stream=None):
    """sfa_decode over a paged cache (pools, page_table and lens as in sfa_kv_append_paged): q, o [B][n][Hq][Dh] bf16,
    lse [B][Hq][n] float32 or None.  An empty slot (lens 0) gives zero rows and LSE -inf.  max_tokens bounds every
    lens[b] (default: what page_table has entries for)."""
    pages, P, Hkv, Dh, B, width = _pool_dims(k_pages, page_table, n)
    if q.dim() != 4:
        raise ValueError("q must be [B][n][Hq][Dh]")
    Hq = q.shape[2]
    T = P * width if max_tokens is None else int(max_tokens)
    st = _tensors(stream, ("q", q, _BF16, (B, n, Hq, Dh)), ("o", o, _BF16, (B, n, Hq, Dh)),
                  ("k_pages", k_pages, _BF16, k_pages.shape), ("v_pages", v_pages, _BF16, k_pages.shape),
                  ("page_table", page_table, _I32, (B, width)), ("lens", lens, _I32, (B,)),
                  _opt("lse", lse, _F32, (B, Hq, n)), _workspace(workspace), _dev_status(dev_status))
    _check(lib().sfa_decode_paged(_p(q), _p(k_pages), _p(v_pages), _p(page_table), _p(lens), _p(o), _p(lse), B, T, pages,
                                  P, width, n, Hq, Hkv, Dh, float(softmax_scale), int(mode), int(window), _p(workspace),
                                  workspace.numel(), _p(dev_status), st), "sfa_decode_paged")
    return o


def hd_pages_workspace_bytes(B, num_pages) -> int:
    return int(lib().hd_pages_workspace_bytes(B, num_pages))


def _page_state(refs, page_table, lens):
    if page_table.dim() != 2:
        raise ValueError("page_table must be [B][max_pages]")
    B, width = page_table.shape
    return B, width, refs.numel(), (("refs", refs, _I32, (refs.numel(),)), ("page_table", page_table, _I32, (B, width)),
                                    ("lens", lens, _I32, (B,)))


def hd_pages_grow(refs, page_table, lens, add, page_tokens, workspace, dev_status=None, stream=None, served=None):
    """lens[b] += add[b], with pages for the new tokens (lowest free ids first, sequences ascending).  refs [num_pages],
    page_table [B][max_pages], lens, add [B] int32.  A sequence that finds no free page stays as it was and sets
    HD_DEVBIT_PAGES; nothing is to be appended to it.  served [B] int32 (written): the tokens each sequence got, add[b]
    or 0, for sfa_kv_append_paged."""
    B, width, pages, state = _page_state(refs, page_table, lens)
    st = _tensors(stream, *state, ("add", add, _I32, (B,)), _opt("served", served, _I32, (B,)), _workspace(workspace),
                  _dev_status(dev_status))
    if served is not None:
        _check(lib().hd_pages_grow_served(_p(refs), _p(page_table), _p(lens), _p(add), _p(served), B, width, pages,
                                          int(page_tokens), _p(workspace), workspace.numel(), _p(dev_status), st),
               "hd_pages_grow_served")
        return
    _check(lib().hd_pages_grow(_p(refs), _p(page_table), _p(lens), _p(add), B, width, pages, int(page_tokens),
                               _p(workspace), workspace.numel(), _p(dev_status), st), "hd_pages_grow")


def hd_pages_fork(refs, page_table, lens, src, dst, tokens, copies, page_tokens, workspace, dev_status=None,
                  stream=None):
    """The empty slots dst get the first `tokens` tokens (None: all) of the slots src: full pages are shared, a partly
    filled last one is new and listed in copies [F][2] (page of src, page of dst; else -1, -1) for hd_pages_copy."""
    B, width, pages, state = _page_state(refs, page_table, lens)
    F = src.numel()
    st = _tensors(stream, *state, ("src", src, _I32, (F,)), ("dst", dst, _I32, (F,)), _opt("tokens", tokens, _I32, (F,)),
                  ("copies", copies, _I32, (F, 2)), _workspace(workspace), _dev_status(dev_status))
    _check(lib().hd_pages_fork(_p(refs), _p(page_table), _p(lens), _p(src), _p(dst), _p(tokens), F, _p(copies), B, width,
                               pages, int(page_tokens), _p(workspace), workspace.numel(), _p(dev_status), st),
           "hd_pages_fork")
    return copies


def hd_pages_free(refs, page_table, lens, seqs, page_tokens, dev_status=None, stream=None):
    """The slots seqs are emptied: lens 0, their entries of page_table -1, their pages held by one sequence less."""
    B, width, pages, state = _page_state(refs, page_table, lens)
    st = _tensors(stream, *state, ("seqs", seqs, _I32, (seqs.numel(),)), _dev_status(dev_status))
    _check(lib().hd_pages_free(_p(refs), _p(page_table), _p(lens), _p(seqs), seqs.numel(), B, width, pages,
                               int(page_tokens), _p(dev_status), st), "hd_pages_free")


def hd_pages_compact(refs, page_table, lens, new_refs, new_table, moves, page_tokens, workspace, dev_status=None,
                     stream=None):
    """The K pages in use get the ids 0 .. K-1 in new_refs and new_table (which may be refs and page_table); moves
    [num_pages // 2][2] lists the pages to copy (old, new; then -1, -1) for hd_pages_copy."""
    B, width, pages, state = _page_state(refs, page_table, lens)
    st = _tensors(stream, *state, ("new_refs", new_refs, _I32, (pages,)), ("new_table", new_table, _I32, (B, width)),
                  ("moves", moves, _I32, (pages // 2, 2)), _workspace(workspace), _dev_status(dev_status))
    _check(lib().hd_pages_compact(_p(refs), _p(page_table), _p(lens), _p(new_refs), _p(new_table), _p(moves), B, width,
                                  pages, int(page_tokens), _p(workspace), workspace.numel(), _p(dev_status),
                                  st), "hd_pages_compact")
    return new_refs, new_table, moves


def hd_pages_copy(k_pages, v_pages, copies, dev_status=None, stream=None):
    """Page copies[i][0] onto page copies[i][1] in both pools (one layer's); pairs of -1 are left out."""
    if k_pages.dim() < 1 or k_pages.shape[0] < 1:
        raise ValueError("k_pages must have a page: [num_pages][page_tokens*n][Hkv][Dh]")
    st = _tensors(stream, ("k_pages", k_pages, _BF16, k_pages.shape), ("v_pages", v_pages, _BF16, k_pages.shape),
                  ("copies", copies, _I32, (copies.numel() // 2, 2)), _dev_status(dev_status))
    _check(lib().hd_pages_copy(_p(k_pages), _p(v_pages), _p(copies), copies.shape[0], k_pages.shape[0],
                               k_pages.numel() // k_pages.shape[0] * 2, _p(dev_status), st), "hd_pages_copy")


# ---- paged cache in 8 bits: the pools hold e4m3 codes [num_pages][Hkv][page_tokens*n][Dh] (torch.float8_e4m3fn), with a
# scale for each block of block_tokens tokens and head, [num_pages][Hkv][page_tokens/block_tokens] (torch.uint8): the
# power of two 2^(byte - 127).

def _q8_pools(k_pages, v_pages, k_scales, v_scales, page_table, n):
    """(num_pages, page_tokens, Hkv, Dh, block_tokens, B, max_pages) and the pools' tensors to check."""
    if k_pages.dim() != 4 or page_table.dim() != 2:
        raise ValueError("k_pages must be [num_pages][Hkv][page_tokens*n][Dh] and page_table [B][max_pages]")
    pages, Hkv, rows, Dh = k_pages.shape
    if n < 1 or rows % n:
        raise ValueError("k_pages.shape[2] must be page_tokens * n")
    P, blocks = rows // n, k_scales.shape[2] if k_scales.dim() == 3 else 0
    if blocks < 1 or P % blocks:
        raise ValueError("k_scales must be [num_pages][Hkv][page_tokens/block_tokens]")
    scales = (pages, Hkv, blocks)
    return (pages, P, Hkv, Dh, P // blocks, *page_table.shape), (
        ("k_pages", k_pages, _F8, k_pages.shape), ("v_pages", v_pages, _F8, k_pages.shape),
        ("k_scales", k_scales, torch.uint8, scales), ("v_scales", v_scales, torch.uint8, scales))


def sfa_kv_append_paged_q8(k_new, v_new, k_pages, v_pages, k_scales, v_scales, page_table, lens, n, offsets=None,
                           dev_status=None, stream=None, served=None):
    """sfa_kv_append_paged into an 8-bit cache: k_new, v_new bf16 [B][n][Hkv][Dh], or with offsets packed rows
    [N*n][Hkv][Dh].  A block's scale is the smallest power of two that holds its new tokens, and at least the one that
    it had if it held tokens before (whose codes are rounded again where it grows)."""
    (pages, P, Hkv, Dh, T, B, width), pools = _q8_pools(k_pages, v_pages, k_scales, v_scales, page_table, n)
    if offsets is None:
        N, shape = B, (B, n, Hkv, Dh)
    else:
        N = k_new.shape[0] // n if k_new.dim() == 3 else 0
        shape = (N * n, Hkv, Dh)
    st = _tensors(stream, ("k_new", k_new, _BF16, shape), ("v_new", v_new, _BF16, shape), *pools,
                  ("page_table", page_table, _I32, (B, width)), ("lens", lens, _I32, (B,)),
                  _opt("offsets", offsets, _I32, (B + 1,)), _opt("served", served, _I32, (B,)), _dev_status(dev_status))
    _check(lib().sfa_kv_append_paged_q8(_p(k_new), _p(v_new), _p(k_pages), _p(v_pages), _p(k_scales), _p(v_scales),
                                        _p(page_table), _p(lens), _p(offsets), _p(served), B, N, pages, P, width, n, Hkv,
                                        Dh, T, _p(dev_status), st), "sfa_kv_append_paged_q8")


def sfa_kv_read_paged_q8(k_pages, v_pages, k_scales, v_scales, page_table, lens, offsets, k, v, n, dev_status=None,
                         stream=None):
    """The values of an 8-bit cache back as packed bf16 rows k, v [N*n][Hkv][Dh] (written, exact): the last
    offsets[b+1] - offsets[b] of the first lens[b] tokens of each sequence.  Rows outside [offsets[0], offsets[B]) are
    left as they were."""
    (pages, P, Hkv, Dh, T, B, width), pools = _q8_pools(k_pages, v_pages, k_scales, v_scales, page_table, n)
    N = k.shape[0] // n if k.dim() == 3 else 0
    shape = (N * n, Hkv, Dh)
    st = _tensors(stream, *pools, ("page_table", page_table, _I32, (B, width)), ("lens", lens, _I32, (B,)),
                  ("offsets", offsets, _I32, (B + 1,)), ("k", k, _BF16, shape), ("v", v, _BF16, shape),
                  _dev_status(dev_status))
    _check(lib().sfa_kv_read_paged_q8(_p(k_pages), _p(v_pages), _p(k_scales), _p(v_scales), _p(page_table), _p(lens),
                                      _p(offsets), _p(k), _p(v), B, N, pages, P, width, n, Hkv, Dh, T, _p(dev_status), st),
           "sfa_kv_read_paged_q8")
    return k, v


def sfa_decode_paged_q8_workspace_bytes(B, max_tokens, n, Hq, Hkv, Dh, mode, window=0) -> int:
    return int(lib().sfa_decode_paged_q8_workspace_bytes(B, max_tokens, n, Hq, Hkv, Dh, int(mode), int(window)))


def sfa_decode_paged_q8(q, k_pages, v_pages, k_scales, v_scales, page_table, lens, o, n, mode, workspace,
                        max_tokens=None, lse=None, softmax_scale=0.0, window=0, dev_status=None, stream=None):
    """sfa_decode_paged over an 8-bit cache: q, o [B][n][Hq][Dh] bf16, lse [B][Hq][n] float32 or None; the result is that
    of the values that the codes stand for, to bounds that hdsfa.h gives (rows with blocks of V, or query values, too far
    apart for them are computed in 32 bits, far slower)."""
    (pages, P, Hkv, Dh, T, B, width), pools = _q8_pools(k_pages, v_pages, k_scales, v_scales, page_table, n)
    if q.dim() != 4:
        raise ValueError("q must be [B][n][Hq][Dh]")
    Hq = q.shape[2]
    most = P * width if max_tokens is None else int(max_tokens)
    st = _tensors(stream, ("q", q, _BF16, (B, n, Hq, Dh)), ("o", o, _BF16, (B, n, Hq, Dh)), *pools,
                  ("page_table", page_table, _I32, (B, width)), ("lens", lens, _I32, (B,)),
                  _opt("lse", lse, _F32, (B, Hq, n)), _workspace(workspace), _dev_status(dev_status))
    _check(lib().sfa_decode_paged_q8(_p(q), _p(k_pages), _p(v_pages), _p(k_scales), _p(v_scales), _p(page_table), _p(lens),
                                     _p(o), _p(lse), B, most, pages, P, width, n, Hq, Hkv, Dh, T, float(softmax_scale),
                                     int(mode), int(window), _p(workspace), workspace.numel(), _p(dev_status), st),
           "sfa_decode_paged_q8")
    return o


def hd_pages_copy_q8(k_pages, v_pages, k_scales, v_scales, copies, dev_status=None, stream=None):
    """hd_pages_copy for an 8-bit cache: codes and scales of page copies[i][0] onto page copies[i][1] in both pools."""
    if k_pages.dim() != 4 or k_scales.dim() != 3 or k_pages.shape[0] < 1:
        raise ValueError("k_pages must be [num_pages][Hkv][page_tokens*n][Dh] and k_scales [num_pages][Hkv][blocks]")
    pages, Hkv = k_pages.shape[:2]
    scales = (pages, Hkv, k_scales.shape[2])
    st = _tensors(stream, ("k_pages", k_pages, _F8, k_pages.shape), ("v_pages", v_pages, _F8, k_pages.shape),
                  ("k_scales", k_scales, torch.uint8, scales), ("v_scales", v_scales, torch.uint8, scales),
                  ("copies", copies, _I32, (copies.numel() // 2, 2)), _dev_status(dev_status))
    _check(lib().hd_pages_copy_q8(_p(k_pages), _p(v_pages), _p(k_scales), _p(v_scales), _p(copies), copies.shape[0], pages,
                                  k_pages.numel() // pages, Hkv * k_scales.shape[2], _p(dev_status), st),
           "hd_pages_copy_q8")


SFA_BWD_NOALLOC_MAX_BYTES = 64 << 20


def sfa_bwd_noalloc(q, k, v, o, lse, dout, dq, dk, dv, n, mode, softmax_scale=0.0, window=0,
                    dev_status=None, stream=None):
    """SFA backward with the library's fixed device workspace (no allocation anywhere,
    at most SFA_BWD_NOALLOC_MAX_BYTES of workspace).  Calls on one device share that
    workspace: order them (one stream, or events) so that none overlap."""
    B, L, Hq, Hkv, Dh = _attn_dims(q, k, n)
    _check(lib().sfa_bwd_noalloc(_p(q), _p(k), _p(v), _p(o), _p(lse), _p(dout), _p(dq), _p(dk),
                                 _p(dv), B, L, n, Hq, Hkv, Dh, float(softmax_scale), int(mode),
                                 int(window), _p(dev_status), _stream(stream)), "sfa_bwd_noalloc")
    return dq, dk, dv


def _wsb(ws):
    return ws.numel() * ws.element_size()


def sfa_bwd_prep(o, dout, lse, n, mode, workspace, Hkv, stream=None):
    """Phase 1 of sfa_bwd: delta = rowsum(dO * O), lse * log2(e), zeroed dQ accumulator."""
    B, nL, Hq, Dh = o.shape
    _check(lib().sfa_bwd_prep(_p(o), _p(dout), _p(lse), B, nL // n, n, Hq, Hkv, Dh, int(mode),
                              _p(workspace), _wsb(workspace), _stream(stream)), "sfa_bwd_prep")


def sfa_bwd_row_terms(o, dout, lse, n, mode, workspace, Hkv, stream=None):
    """The delta / lse half of sfa_bwd_prep (no zeroing of the dQ accumulator)."""
    B, nL, Hq, Dh = o.shape
    _check(lib().sfa_bwd_row_terms(_p(o), _p(dout), _p(lse), B, nL // n, n, Hq, Hkv, Dh, int(mode),
                                   _p(workspace), _wsb(workspace), _stream(stream)), "sfa_bwd_row_terms")


def sfa_bwd_clear(B, L, n, Hq, Hkv, Dh, mode, workspace, stream=None):
    """The other half: zero the workspace's fp32 dQ accumulator (independent of the forward)."""
    _check(lib().sfa_bwd_clear(B, L, n, Hq, Hkv, Dh, int(mode), _p(workspace), _wsb(workspace),
                               _stream(stream)), "sfa_bwd_clear")


def sfa_bwd_main(q, k, v, dout, dk, dv, n, mode, workspace, softmax_scale=0.0, window=0,
                 dev_status=None, stream=None):
    """Phase 2 of sfa_bwd: dK, dV and the fp32 dQ accumulator."""
    B, L, Hq, Hkv, Dh = _attn_dims(q, k, n)
    _check(lib().sfa_bwd_main(_p(q), _p(k), _p(v), _p(dout), _p(dk), _p(dv), B, L, n, Hq, Hkv, Dh,
                              float(softmax_scale), int(mode), int(window), _p(workspace),
                              _wsb(workspace), _p(dev_status), _stream(stream)), "sfa_bwd_main")


def sfa_bwd_finalize(dq, n, mode, workspace, Hkv, softmax_scale=0.0, stream=None):
    """Phase 3 of sfa_bwd: dq = bf16(scale * accumulator)."""
    B, nL, Hq, Dh = dq.shape
    _check(lib().sfa_bwd_finalize(_p(dq), B, nL // n, n, Hq, Hkv, Dh, float(softmax_scale), int(mode),
                                  _p(workspace), _wsb(workspace), _stream(stream)), "sfa_bwd_finalize")
