"""BAPS attention on MI355X: Python binding of libbaps.so.

The names match the C ABI in include/baps.h.  This module only marshals
arguments (tensor -> device pointer, stream -> handle, status -> exception);
every step of the method runs in the library's HIP kernels.  PyTorch is used
for device memory and streams only.  If the library has not been built the
calls raise: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbaps.so")

BAPS_OK = 0
BAPS_INVALID_ARGUMENT = 1
BAPS_UNSUPPORTED = 2
BAPS_HIP_ERROR = 3
BAPS_HIF8_SATURATE = 1
BAPS_HIF8_TIES_EVEN = 2
BAPS_TIES_AWAY = 0
BAPS_TIES_EVEN = 1

BAPS_SPLIT_SCRATCH_BYTES = 32 << 20

EXPORTS = ("baps_attention_fwd", "baps_attention_fwd_ex", "baps_attention_fwd_split", "baps_attention_fwd_dump",
           "baps_attention_fwd_split_noalloc",
           "hif8_encode", "hif8_decode", "baps_softmax_block", "baps_get_exp2_lut", "baps_init",
           "baps_attention_window", "baps_cache_append", "baps_cache_attention", "baps_cache_fork", "baps_cache_compact",
           "baps_attention_split_workspace", "baps_attention_window_workspace", "baps_cache_attention_workspace",
           "baps_cache_pages_workspace",
           "baps_last_hip_error", "baps_status_string")

_lib = None


class BapsError(RuntimeError):
    def __init__(self, fn, status):
        detail = f", {load().baps_last_hip_error().decode()}" if status == 3 else ""
        super().__init__(f"{fn}: {status_string(status)} (status {status}{detail})")
        self.status = status


class baps_params_t(ctypes.Structure):
    _fields_ = [("lambda_", ctypes.c_int), ("n_b0", ctypes.c_int), ("scale_log2", ctypes.c_float),
                ("restart_counts", ctypes.c_void_p), ("mode", ctypes.c_int), ("restart_rows", ctypes.c_int),
                ("b0_last", ctypes.c_int), ("tile_counts", ctypes.c_void_p), ("qk_format", ctypes.c_int),
                ("q_scale", ctypes.c_float), ("k_scale", ctypes.c_float), ("tie_mode", ctypes.c_int),
                ("saturate", ctypes.c_int), ("out_bf16", ctypes.c_int)]


class baps_cache_t(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("layers", ctypes.c_int), ("num_pages", ctypes.c_int), ("Hkv", ctypes.c_int), ("page", ctypes.c_int),
                ("D", ctypes.c_int)]


# softmax setups (include/baps.h)
BAPS_MODE_E2E_HIF8 = 0
BAPS_MODE_DEFAULT = 1
BAPS_MODE_EXP2_HIF8 = 2
# Q/K formats (include/baps.h)
BAPS_QK_BF16 = 0
BAPS_QK_FP8_E4M3 = 1


def load():
    """Load libbaps.so (raises when it is missing: build it first)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run __graft_entry__.build() (hipcc, gfx950) first")
    # torch ships its own HIP and HSA runtimes under the same sonames as the
    # system ones; with torch loaded first the library binds to them, so the
    # process holds one runtime (two would both claim the GPU, and the second
    # to start up finds no device).
    import torch  # noqa: F401
    L = ctypes.CDLL(LIB_PATH)
    P, I, LL = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong
    L.baps_attention_fwd.argtypes = [P, P, P, P, P, I, I, I, I, I, I, I, I, P]
    L.baps_attention_fwd_ex.argtypes = [P, P, P, P, P, I, I, I, I, I, I, I, I,
                                        ctypes.POINTER(baps_params_t), P]
    L.baps_attention_fwd_split.argtypes = [P, P, P, P, P, I, I, I, I, I, I, I, I,
                                           ctypes.POINTER(baps_params_t), P, LL, P]
    L.baps_attention_fwd_dump.argtypes = [P, P, P, P, P, I, I, I, I, I, I, I, I,
                                          ctypes.POINTER(baps_params_t), P, P, P, P]
    L.baps_attention_fwd_split_noalloc.argtypes = [P, P, P, P, P, I, I, I, I, I, I, I, I,
                                                   ctypes.POINTER(baps_params_t), P]
    L.baps_attention_split_workspace.argtypes = [I, I, I, I, I, I, I, ctypes.POINTER(baps_params_t)]
    L.baps_attention_window.argtypes = [P, P, P, P, P, I, I, I, I, I, I, I, I, I, ctypes.POINTER(baps_params_t), P, LL, P]
    L.baps_attention_window_workspace.argtypes = [I, I, I, I, I, I, I, I, I, ctypes.POINTER(baps_params_t)]
    C = ctypes.POINTER(baps_cache_t)
    L.baps_cache_append.argtypes = [C, I, P, P, LL, P, P, P, I, I, I, I, P]
    L.baps_cache_attention.argtypes = [C, I, P, LL, P, P, P, P, P, I, I, I, I, I, I, I, I, ctypes.c_float, P, LL, P]
    L.baps_cache_attention_workspace.argtypes = [C, I, I, I, I, I, I, I]
    L.baps_cache_fork.argtypes = [C, P, P, P, I, P, P, I, I, P, P, P, P, P, LL, P]
    L.baps_cache_compact.argtypes = [C, P, LL, P, P, P, P, P, P, LL, P]
    L.baps_cache_pages_workspace.argtypes = [I, I]
    L.hif8_encode.argtypes = [P, P, LL, I, P]
    L.hif8_decode.argtypes = [P, P, LL, P]
    L.baps_softmax_block.argtypes = [P, LL, LL, LL, I, I, I, I, P, P, P, P, P, P]
    L.baps_get_exp2_lut.argtypes = [P]
    L.baps_init.argtypes = []
    L.baps_status_string.argtypes = [I]
    L.baps_status_string.restype = ctypes.c_char_p
    L.baps_last_hip_error.argtypes = []
    L.baps_last_hip_error.restype = ctypes.c_char_p
    for name in EXPORTS[:-2]:
        getattr(L, name).restype = I
    L.baps_attention_split_workspace.restype = LL
    L.baps_attention_window_workspace.restype = LL
    L.baps_cache_attention_workspace.restype = LL
    L.baps_cache_pages_workspace.restype = LL
    _lib = L
    return L


def status_string(status: int) -> str:
    return load().baps_status_string(int(status)).decode()


def _p(x):
    """Device pointer of a tensor (or an int / None passed through)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream):
    if stream is None:
        # The current stream of the current device.  torch.cuda.current_stream()
        # builds a Stream object around the same handle: 2.9 us of a call that
        # took 12.5 us in all with it; the lookup of the handle (not part of
        # torch's public interface) takes 0.3.
        import torch
        try:
            if torch.cuda.is_initialized():
                return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            pass
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(fn, st):
    if st != BAPS_OK:
        raise BapsError(fn, st)


def baps_attention_fwd(q, k, v, o, lse, B, Hq, Hkv, Sq, Sk, D, causal, block, stream=None):
    _check("baps_attention_fwd", load().baps_attention_fwd(
        _p(q), _p(k), _p(v), _p(o), _p(lse), B, Hq, Hkv, Sq, Sk, D, int(causal), block, _stream(stream)))


def _params(lam=1, n_b0=1, scale_log2=0.0, restart_counts=None, mode=BAPS_MODE_E2E_HIF8, restart_rows=1,
            b0_last=False, tile_counts=None, qk_scales=None, tie_mode=BAPS_TIES_AWAY, saturate=True,
            out_bf16=False):
    fmt, qs, ks = (BAPS_QK_BF16, 1.0, 1.0) if qk_scales is None else (BAPS_QK_FP8_E4M3,) + tuple(qk_scales)
    return baps_params_t(int(lam), int(n_b0), float(scale_log2), _p(restart_counts), int(mode), int(restart_rows),
                         int(bool(b0_last)), _p(tile_counts), int(fmt), float(qs), float(ks), int(tie_mode),
                         int(bool(saturate)), int(bool(out_bf16)))


def baps_attention_fwd_ex(q, k, v, o, lse, B, Hq, Hkv, Sq, Sk, D, causal, block, lam=1, n_b0=1,
                          scale_log2=0.0, restart_counts=None, stream=None, mode=BAPS_MODE_E2E_HIF8,
                          restart_rows=1, b0_last=False, tile_counts=None, qk_scales=None, tie_mode=BAPS_TIES_AWAY,
                          saturate=True, out_bf16=False):
    """qk_scales=(q_scale, k_scale): q and k are FP8 E4M3 codes (uint8 tensors).
    out_bf16: o is a bf16 tensor."""
    prm = _params(lam, n_b0, scale_log2, restart_counts, mode, restart_rows, b0_last, tile_counts, qk_scales,
                  tie_mode, saturate, out_bf16)
    _check("baps_attention_fwd_ex", load().baps_attention_fwd_ex(
        _p(q), _p(k), _p(v), _p(o), _p(lse), B, Hq, Hkv, Sq, Sk, D, int(causal), block,
        ctypes.byref(prm), _stream(stream)))


def baps_attention_fwd_dump(q, k, v, o, lse, B, Hq, Hkv, Sq, Sk, D, causal, block, row_slot, acc_out, ref_out,
                            stream=None, **knobs):
    """The fused pass with a dump of the selected rows' raw dot products and
    block references (include/baps.h); knobs as baps_attention_fwd_ex."""
    prm = _params(**knobs)
    _check("baps_attention_fwd_dump", load().baps_attention_fwd_dump(
        _p(q), _p(k), _p(v), _p(o), _p(lse), B, Hq, Hkv, Sq, Sk, D, int(causal), block,
        ctypes.byref(prm), _p(row_slot), _p(acc_out), _p(ref_out), _stream(stream)))


def baps_attention_split_workspace(B, Hq, Hkv, Sq, Sk, D, block, lam=1, n_b0=1, scale_log2=0.0,
                                   mode=BAPS_MODE_E2E_HIF8, restart_rows=1, b0_last=False, qk_scales=None,
                                   tie_mode=BAPS_TIES_AWAY, saturate=True, out_bf16=False):
    prm = _params(lam, n_b0, scale_log2, None, mode, restart_rows, b0_last, None, qk_scales, tie_mode, saturate,
                  out_bf16)
    return int(load().baps_attention_split_workspace(B, Hq, Hkv, Sq, Sk, D, block, ctypes.byref(prm)))


def baps_attention_fwd_split(q, k, v, o, lse, B, Hq, Hkv, Sq, Sk, D, causal, block, workspace, workspace_bytes,
                             lam=1, n_b0=1, scale_log2=0.0, restart_counts=None, stream=None,
                             mode=BAPS_MODE_E2E_HIF8, restart_rows=1, b0_last=False, tile_counts=None,
                             qk_scales=None, tie_mode=BAPS_TIES_AWAY, saturate=True, out_bf16=False):
    prm = _params(lam, n_b0, scale_log2, restart_counts, mode, restart_rows, b0_last, tile_counts, qk_scales,
                  tie_mode, saturate, out_bf16)
    _check("baps_attention_fwd_split", load().baps_attention_fwd_split(
        _p(q), _p(k), _p(v), _p(o), _p(lse), B, Hq, Hkv, Sq, Sk, D, int(causal), block,
        ctypes.byref(prm), _p(workspace), int(workspace_bytes), _stream(stream)))


def baps_attention_fwd_split_noalloc(q, k, v, o, lse, B, Hq, Hkv, Sq, Sk, D, causal, block, stream=None, **knobs):
    """The split-key path on the library's static scratch (no allocation);
    knobs as baps_attention_fwd_ex."""
    prm = _params(**knobs)
    _check("baps_attention_fwd_split_noalloc", load().baps_attention_fwd_split_noalloc(
        _p(q), _p(k), _p(v), _p(o), _p(lse), B, Hq, Hkv, Sq, Sk, D, int(causal), block,
        ctypes.byref(prm), _stream(stream)))


def hif8_encode(x, codes, n, flags=BAPS_HIF8_SATURATE, stream=None):
    _check("hif8_encode", load().hif8_encode(_p(x), _p(codes), n, flags, _stream(stream)))


def hif8_decode(codes, x, n, stream=None):
    _check("hif8_decode", load().hif8_decode(_p(codes), _p(x), n, _stream(stream)))


def baps_softmax_block(s, rows, cols, ld_s, block, lam, n_b0, flags, p_codes, ref_shift, m_final, d_final,
                       restarted=None, stream=None):
    _check("baps_softmax_block", load().baps_softmax_block(
        _p(s), rows, cols, ld_s, block, lam, n_b0, flags, _p(p_codes), _p(ref_shift), _p(m_final),
        _p(d_final), _p(restarted), _stream(stream)))


def baps_attention_window_workspace(B, Hq, Hkv, Sq, Sk, D, window, sinks, block, **knobs):
    """knobs as baps_attention_fwd_ex."""
    prm = _params(**knobs)
    return int(load().baps_attention_window_workspace(B, Hq, Hkv, Sq, Sk, D, window, sinks, block, ctypes.byref(prm)))


def baps_attention_window(q, k, v, o, lse, B, Hq, Hkv, Sq, Sk, D, window, sinks, block, workspace=None, workspace_bytes=0,
                          stream=None, **knobs):
    """knobs as baps_attention_fwd_ex."""
    prm = _params(**knobs)
    _check("baps_attention_window", load().baps_attention_window(
        _p(q), _p(k), _p(v), _p(o), _p(lse), B, Hq, Hkv, Sq, Sk, D, window, sinks, block, ctypes.byref(prm),
        _p(workspace), int(workspace_bytes), _stream(stream)))


def baps_cache_append(cache, layer, k, v, token_stride, cu_new, lens, table, table_width, B, total_new, max_new,
                      stream=None):
    _check("baps_cache_append", load().baps_cache_append(
        ctypes.byref(cache), layer, _p(k), _p(v), token_stride, _p(cu_new), _p(lens), _p(table), table_width, B,
        total_new, max_new, _stream(stream)))


def baps_cache_attention_workspace(cache, B, Hq, total_q, max_q, max_len, window=0, sinks=0):
    return int(load().baps_cache_attention_workspace(ctypes.byref(cache), B, Hq, total_q, max_q, max_len, window, sinks))


def baps_cache_attention(cache, layer, q, q_stride, o, lse, cu_q, lens, table, table_width, B, Hq, total_q, max_q, max_len,
                         window=0, sinks=0, scale_log2=0.0, workspace=None, workspace_bytes=0, stream=None):
    _check("baps_cache_attention", load().baps_cache_attention(
        ctypes.byref(cache), layer, _p(q), q_stride, _p(o), _p(lse), _p(cu_q), _p(lens), _p(table), table_width, B, Hq,
        total_q, max_q, max_len, window, sinks, scale_log2, _p(workspace), int(workspace_bytes), _stream(stream)))


def baps_cache_pages_workspace(num_pages, B_out):
    return int(load().baps_cache_pages_workspace(num_pages, B_out))


def baps_cache_fork(cache, table_in, lens_in, refs_in, B_in, parent, grow, B_out, table_width, table_out, lens_out, refs_out,
                    missing, workspace, workspace_bytes, stream=None):
    _check("baps_cache_fork", load().baps_cache_fork(
        ctypes.byref(cache), _p(table_in), _p(lens_in), _p(refs_in), B_in, _p(parent), _p(grow), B_out, table_width,
        _p(table_out), _p(lens_out), _p(refs_out), _p(missing), _p(workspace), int(workspace_bytes), _stream(stream)))


def baps_cache_compact(cache, table_in, entries, refs_in, table_out, refs_out, remap, live, workspace, workspace_bytes,
                       stream=None):
    _check("baps_cache_compact", load().baps_cache_compact(
        ctypes.byref(cache), _p(table_in), entries, _p(refs_in), _p(table_out), _p(refs_out), _p(remap), _p(live),
        _p(workspace), int(workspace_bytes), _stream(stream)))


def baps_get_exp2_lut():
    buf = (ctypes.c_ubyte * 256)()
    _check("baps_get_exp2_lut", load().baps_get_exp2_lut(buf))
    return bytes(buf)


def baps_init():
    _check("baps_init", load().baps_init())


# ------------------------------------------------------------ tensor helpers
def attention(q, k, v, causal, block, lse=True, lam=None, n_b0=None, scale_log2=0.0, restart_counts=None,
              stream=None, mode=BAPS_MODE_E2E_HIF8, split=False, restart_rows=1, b0_last=False, tile_counts=None,
              qk_scales=None, tie_mode=BAPS_TIES_AWAY, saturate=True, out_bf16=False):
    """Allocate O (and lse) with torch on q's device and run the fused pass.
    q [B,Hq,Sq,D], k/v [B,Hkv,Sk,D] bf16 CUDA tensors, contiguous.  split:
    take baps_attention_fwd_split, with a workspace allocated here.
    restart_rows / b0_last / tile_counts: the tile-level restart knobs of
    baps_params_t.  qk_scales=(q_scale, k_scale): q and k are FP8 E4M3 codes
    (uint8 tensors) with those dequantisation scales.  out_bf16: O is
    returned as bf16."""
    import torch
    B, Hq, Sq, D = q.shape
    Hkv, Sk = k.shape[1], k.shape[2]
    _check_inputs(q, k, v, qk_scales)
    o = torch.empty((B, Hq, Sq, D), dtype=torch.bfloat16 if out_bf16 else torch.float32, device=q.device)
    l = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device) if lse else None
    lam_, nb_ = 1 if lam is None else lam, 1 if n_b0 is None else n_b0
    extra = dict(tie_mode=tie_mode, saturate=saturate, out_bf16=out_bf16)
    if split:
        nbytes = baps_attention_split_workspace(B, Hq, Hkv, Sq, Sk, D, block, lam_, nb_, scale_log2, mode,
                                                restart_rows, b0_last, qk_scales, **extra)
        ws = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=q.device)
        baps_attention_fwd_split(q, k, v, o, l, B, Hq, Hkv, Sq, Sk, D, causal, block, ws, nbytes, lam_, nb_,
                                 scale_log2, restart_counts, stream, mode, restart_rows, b0_last, tile_counts,
                                 qk_scales, **extra)
    elif (lam is None and n_b0 is None and not scale_log2 and restart_counts is None and mode == BAPS_MODE_E2E_HIF8
          and restart_rows == 1 and not b0_last and tile_counts is None and qk_scales is None
          and tie_mode == BAPS_TIES_AWAY and saturate and not out_bf16):
        baps_attention_fwd(q, k, v, o, l, B, Hq, Hkv, Sq, Sk, D, causal, block, stream)
    else:
        baps_attention_fwd_ex(q, k, v, o, l, B, Hq, Hkv, Sq, Sk, D, causal, block, lam_, nb_, scale_log2,
                              restart_counts, stream, mode, restart_rows, b0_last, tile_counts, qk_scales, **extra)
    return o, l


def attention_window(q, k, v, window, sinks=0, block=128, lse=True, stream=None, out_bf16=False, **knobs):
    """Attention with a sliding window and sink tokens (baps_attention_window):
    allocates O (and lse) and the workspace with torch.  q [B,Hq,Sq,D], k/v
    [B,Hkv,Sk,D] bf16 device tensors, contiguous; knobs as
    baps_attention_fwd_ex (mode, lam, n_b0, scale_log2, b0_last, ...)."""
    import torch
    B, Hq, Sq, D = q.shape
    Hkv, Sk = k.shape[1], k.shape[2]
    _check_inputs(q, k, v, None)
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != D or not q.device == k.device == v.device:
        raise ValueError("k and v must be [B, Hkv, Sk, D] for q [B, Hq, Sq, D], on one device")
    o = torch.empty((B, Hq, Sq, D), dtype=torch.bfloat16 if out_bf16 else torch.float32, device=q.device)
    l = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device) if lse else None
    prm = _params(out_bf16=out_bf16, **knobs)

    def run():
        nbytes = int(load().baps_attention_window_workspace(B, Hq, Hkv, Sq, Sk, D, window, sinks, block, ctypes.byref(prm)))
        ws = _scratch(nbytes, q.device, stream)
        _check("baps_attention_window", load().baps_attention_window(
            _p(q), _p(k), _p(v), _p(o), _p(l), B, Hq, Hkv, Sq, Sk, D, window, sinks, block, ctypes.byref(prm), _p(ws), nbytes,
            _stream(stream)))
    guard = _on_device(q.device)
    if guard is None:
        run()
    else:
        with guard:
            run()
    return o, l


def _check_inputs(q, k, v, qk_scales):
    import torch
    qk_dtype = torch.bfloat16 if qk_scales is None else torch.uint8
    for t, dt in ((q, qk_dtype), (k, qk_dtype), (v, torch.bfloat16)):
        if t.dtype != dt or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("q, k (bf16, or uint8 FP8 codes with qk_scales) and v (bf16) must be contiguous "
                             "device tensors")


def attention_dump(q, k, v, causal, block, rows, lam=1, n_b0=1, scale_log2=0.0, mode=BAPS_MODE_E2E_HIF8,
                   restart_rows=1, b0_last=False, qk_scales=None, tie_mode=BAPS_TIES_AWAY, saturate=True,
                   stream=None):
    """baps_attention_fwd_dump with buffers allocated here: the fused pass
    (o, lse as from attention()) plus, for the global query rows `rows`
    ((b*Hq + h)*Sq + r, distinct), their raw dot products acc [n, Sk] (NaN
    where the row sees no key) and block references ref [n, ceil(Sk/block)]
    (NaN where the row sees no key of the block), as device tensors."""
    import torch
    B, Hq, Sq, D = q.shape
    Hkv, Sk = k.shape[1], k.shape[2]
    _check_inputs(q, k, v, qk_scales)
    rows = torch.as_tensor(rows, dtype=torch.int64).reshape(-1)
    n = rows.numel()
    if n and (rows.min() < 0 or rows.max() >= B * Hq * Sq or rows.unique().numel() != n):
        raise ValueError("rows must be distinct query-row indices")
    slot = torch.full((B * Hq * Sq,), -1, dtype=torch.int32)
    slot[rows] = torch.arange(n, dtype=torch.int32)
    slot = slot.to(q.device)
    nblk = (Sk + block - 1) // block
    acc = torch.full((max(n, 1), max(Sk, 1)), float("nan"), dtype=torch.float32, device=q.device)
    ref = torch.full((max(n, 1), max(nblk, 1)), float("nan"), dtype=torch.float32, device=q.device)
    o = torch.empty((B, Hq, Sq, D), dtype=torch.float32, device=q.device)
    l = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device)
    baps_attention_fwd_dump(q, k, v, o, l, B, Hq, Hkv, Sq, Sk, D, causal, block, slot, acc, ref, stream,
                            lam=lam, n_b0=n_b0, scale_log2=scale_log2, mode=mode, restart_rows=restart_rows,
                            b0_last=b0_last, qk_scales=qk_scales, tie_mode=tie_mode, saturate=saturate)
    return o, l, acc[:n, :Sk], ref[:n, :nblk]


def _on_device(device):
    """A guard that makes `device` the current one (None where it is already)."""
    import torch
    return None if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _scratch(nbytes, device, stream):
    """A workspace that the caching allocator keeps from others until the call's stream is past it."""
    import torch
    if not nbytes:
        return None
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if stream is not None:
        ws.record_stream(torch.cuda.ExternalStream(_stream(stream), device=device))
    return ws


class PagedCache:
    """A paged 8-bit key/value cache over tensors of the caller (include/baps.h
    states the layout): k [layers, num_pages, Hkv, page, D] and v [layers,
    num_pages, Hkv, page // 16, D, 16], FP8 E4M3 codes as uint8; k_exp, v_exp
    [layers, num_pages, Hkv], the scales' exponents as uint8.  Index tensors
    are int32 on the cache's device; outputs are allocated with torch."""

    def __init__(self, k, v, k_exp, v_exp):
        import torch
        if k.dim() != 5:
            raise ValueError("k must be [layers, num_pages, Hkv, page, D]")
        layers, pages, Hkv, page, D = k.shape
        for name, t, shape in (("k", k, k.shape), ("v", v, (layers, pages, Hkv, page // 16, D, 16)),
                               ("k_exp", k_exp, (layers, pages, Hkv)), ("v_exp", v_exp, (layers, pages, Hkv))):
            if t.dtype != torch.uint8 or not t.is_contiguous() or not t.is_cuda or t.device != k.device:
                raise ValueError(f"{name} must be a contiguous uint8 device tensor (all four on one device)")
            if tuple(t.shape) != tuple(shape):
                raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
        if D not in (64, 128) or page not in (16, 32, 64, 128):
            raise ValueError("D must be 64 or 128 and page 16, 32, 64 or 128")
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.layers, self.num_pages, self.Hkv, self.page, self.D = layers, pages, Hkv, page, D
        self.device = k.device
        self._int32, self._bf16, self._float32 = torch.int32, torch.bfloat16, torch.float32
        self.c = baps_cache_t(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(), layers, pages, Hkv, page, D)

    @classmethod
    def zeros(cls, layers, num_pages, Hkv, page, D, device="cuda"):
        import torch
        z = lambda *s: torch.zeros(s, dtype=torch.uint8, device=device)  # noqa: E731
        return cls(z(layers, num_pages, Hkv, page, D), z(layers, num_pages, Hkv, page // 16, D, 16),
                   z(layers, num_pages, Hkv), z(layers, num_pages, Hkv))

    def _ints(self, name, t, dim, n=None):
        if t.dtype != self._int32 or not t.is_contiguous() or t.device != self.device or t.dim() != dim:
            raise ValueError(f"{name} must be a contiguous int32 tensor of {dim} dimension(s) on {self.device}")
        if n is not None and t.shape[0] != n:
            raise ValueError(f"{name} must have {n} rows, not {t.shape[0]}")

    def _sequences(self, name, cu, lens, table):
        """Checks the arrays of a batch; returns its size."""
        B = lens.shape[0]
        self._ints("lens", lens, 1)
        self._ints(name, cu, 1, B + 1)
        self._ints("table", table, 2, B)
        return B

    def _rows(self, name, t, heads):
        """Packed bf16 rows [T, heads, D], the heads of a row next to each other; returns the row stride."""
        shape, stride = t.shape, t.stride()
        if (len(shape) != 3 or shape[1] != heads or shape[2] != self.D or t.dtype != self._bf16 or t.device != self.device
                or stride[2] != 1 or (heads > 1 and stride[1] != self.D)):
            raise ValueError(f"{name} must be bf16 [T, {heads}, {self.D}] on {self.device} with contiguous rows")
        return stride[0] if shape[0] > 1 else heads * self.D

    def _call(self, fn, *args):
        guard = _on_device(self.device)
        if guard is None:
            return fn(self.c, *args)
        with guard:
            return fn(self.c, *args)

    def append(self, layer, k, v, cu_new, lens, table, max_new, stream=None):
        """k, v [T, Hkv, D] bf16: the new tokens of every sequence, packed (rows may be strided, both alike)."""
        B = self._sequences("cu_new", cu_new, lens, table)
        stride = self._rows("k", k, self.Hkv)
        if self._rows("v", v, self.Hkv) != stride or k.shape[0] != v.shape[0]:
            raise ValueError("k and v must have the same rows and row stride")
        self._call(baps_cache_append, layer, k, v, stride, cu_new, lens, table, table.shape[1], B, k.shape[0], max_new, stream)

    def attention(self, layer, q, cu_q, lens, table, max_q, max_len, window=0, sinks=0, scale_log2=0.0, lse=True,
                  stream=None):
        """q [T, Hq, D] bf16, packed (rows may be strided); returns o [T, Hq, D] bf16 and lse [T, Hq] (or None)."""
        B = self._sequences("cu_q", cu_q, lens, table)
        T, Hq = q.shape[0], q.shape[1]
        stride = self._rows("q", q, Hq)
        o = q.new_empty((T, Hq, self.D))
        l = q.new_empty((T, Hq), dtype=self._float32) if lse else None

        def run(c):
            nbytes = baps_cache_attention_workspace(c, B, Hq, T, max_q, max_len, window, sinks)
            baps_cache_attention(c, layer, q, stride, o, l, cu_q, lens, table, table.shape[1], B, Hq, T, max_q, max_len,
                                 window, sinks, scale_log2, _scratch(nbytes, self.device, stream), nbytes, stream)
        self._call(run)
        return o, l

    def _int_outputs(self, nbytes, *sizes, stream):
        """A workspace of nbytes and int32 outputs, parts of one allocation (one costs the host as much as a small kernel)."""
        ws, *outs = self.k_exp.new_empty(nbytes // 4 + sum(sizes), dtype=self._int32).split_with_sizes((nbytes // 4, *sizes))
        if stream is not None:
            import torch
            ws.record_stream(torch.cuda.ExternalStream(_stream(stream), device=self.device))
        return ws, *outs

    def fork(self, table, lens, refs, parent, grow=None, stream=None):
        """The next set of sequences: (table, lens, refs, missing), new tensors; the pool's copies are made in place."""
        B_in, B_out = lens.shape[0], parent.shape[0]
        self._ints("lens", lens, 1)
        self._ints("table", table, 2, B_in)
        self._ints("refs", refs, 1, self.num_pages)
        self._ints("parent", parent, 1)
        if grow is not None:
            self._ints("grow", grow, 1, B_out)
        width = table.shape[1]
        nbytes = baps_cache_pages_workspace(0, B_out)
        ws, out, lens_out, refs_out, missing = self._int_outputs(nbytes, B_out * width, B_out, self.num_pages, 1, stream=stream)
        self._call(baps_cache_fork, table, lens, refs, B_in, parent, grow, B_out, width, out, lens_out, refs_out, missing, ws,
                   nbytes, stream)
        return out.view(B_out, width), lens_out, refs_out, missing

    def compact(self, table, refs, stream=None):
        """(table, refs, remap, live), new tensors; the pool's pages are moved in place."""
        self._ints("table", table, 2)
        self._ints("refs", refs, 1, self.num_pages)
        n = self.num_pages
        nbytes = baps_cache_pages_workspace(n, 0)
        ws, out, refs_out, remap, live = self._int_outputs(nbytes, table.numel(), n, n, 1, stream=stream)
        self._call(baps_cache_compact, table, table.numel(), refs, out, refs_out, remap, live, ws, nbytes, stream)
        return out.view(table.shape), refs_out, remap, live
