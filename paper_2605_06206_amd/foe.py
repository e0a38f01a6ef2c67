"""Thin Python binding of ``libfoe.so`` (C ABI in ``include/foe.h``).

Argument marshalling only: tensors are passed as device pointers plus the
current HIP stream, and every step of the block runs in the library's HIP
kernels.  PyTorch provides device memory and streams.  There is no fallback:
if the library is missing or a tensor is not a contiguous GPU tensor of the
right dtype, the call raises.
"""

from __future__ import annotations

import ctypes
import os

import torch

F32 = 0
BF16 = 1
GATE_RENORM = 0   # foe_gating
GATE_GLOBAL = 1

FOE_OK = 0
FOE_ERR_INVALID = -1
FOE_ERR_UNSUPPORTED = -2
FOE_ERR_WORKSPACE = -3
FOE_ERR_HIP = -4

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfoe.so")

_c_int, _c_float, _c_size = ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_p = ctypes.c_void_p

_SIGNATURES = {
    "foe_route": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _p, _p, _p, _p, _p, _p]),
    "foe_route_ex": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _p, _p,
                              _p, _p, _p]),
    "foe_permute": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _p, _p, _p, _p, _p, _p, _p,
                             _p, _c_size, _p]),
    "foe_expert_ffn": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _p, _p, _p, _p, _p, _p,
                                _p, _c_size, _p]),
    "foe_combine": (_c_int, [_c_int, _c_int, _c_int, _c_int, _p, _p, _p, _p, _p, _p]),
    "foe_reduce": (_c_int, [_c_int, _c_int, _c_int, _c_int, _p, _p, _c_float, _p, _p]),
    "foe_cluster_block": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _p,
                                   _p, _p, _p, _p, _c_float, _p, _p, _c_size, _p]),
    "foe_cluster_block_ex": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int,
                                      _c_int, _p, _p, _p, _p, _p, _p, _c_float, _p, _p, _c_size,
                                      _p]),
    "foe_cluster_block_noalloc": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_int,
                                           _c_int, _p, _p, _p, _p, _p, _p, _c_float, _p, _p]),
    "foe_workspace_bytes": (_c_size, [ctypes.c_char_p, _c_int, _c_int, _c_int, _c_int, _c_int,
                                      _c_int, _c_int]),
    "foe_group_attention": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_float,
                                     _c_float, _p, _p, _p, _p, _p, _c_size, _p]),
    "foe_group_attention_workspace_bytes": (_c_size, [_c_int, _c_int, _c_int, _c_int, _c_int]),
    "foe_cache_append": (_c_int, [_c_int] * 8 + [_c_float] * 2 + [_p] * 10),
    "foe_cache_attention": (_c_int, [_c_int] * 9 + [_p] * 10 + [_p, _c_size, _p]),
    "foe_cache_attention_workspace_bytes": (_c_size, [_c_int] * 8),
    "foe_cache_evict": (_c_int, [_c_int] * 7 + [_p] * 3 + [_c_int] + [_p] * 7 +
                        [_c_size, _p]),
    "foe_cache_evict_workspace_bytes": (_c_size, [_c_int] * 3),
    "foe_last_error": (ctypes.c_char_p, []),
    "foe_profile_enable": (_c_int, [_c_int]),
    "foe_profile_reset": (_c_int, []),
    "foe_profile_kernel": (_c_int, [ctypes.c_char_p, ctypes.POINTER(_c_int),
                                    ctypes.POINTER(ctypes.c_double)]),
    "foe_profile_names": (_c_int, [ctypes.c_char_p, _c_size]),
}

_lib = None


class FoeError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"[status {status}] {msg}")
        self.status = status


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2605_06206_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def last_error():
    return lib().foe_last_error().decode()


def _check(rc, name):
    if rc != FOE_OK:
        raise FoeError(rc, f"{name}: {last_error()}")


def _dt(t):
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype} (bf16 or fp32)")


def _dev(t, name, dtype=None):
    """Device pointer of a contiguous GPU tensor (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def workspace_bytes(op, dt, C=0, T=0, d=0, E=0, k=0, F=0):
    n = lib().foe_workspace_bytes(op.encode(), dt, C, T, d, E, k, F)
    if n == ctypes.c_size_t(-1).value:
        raise FoeError(FOE_ERR_INVALID, f"foe_workspace_bytes({op}): {last_error()}")
    return n


def _workspace(ws, nbytes, device):
    if ws is None or ws.numel() < nbytes:
        ws = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
    return ws


def _gating(gating):
    codes = {"renorm": GATE_RENORM, "global": GATE_GLOBAL}
    if gating not in codes:
        raise ValueError(f"gating must be 'renorm' or 'global', got {gating!r}")
    return codes[gating]


def route(x, w_router, bias, k, topk_idx=None, topk_w=None, stream=None, gating="renorm"):
    """foe_route (w_router [E,d]) or foe_route_ex (w_router [G,E,d], or a
    gating other than "renorm"): returns (topk_idx, topk_w), [T,k] or [G,T,k]."""
    T, d = x.shape
    grouped = w_router.dim() == 3
    G = w_router.shape[0] if grouped else 1
    E = w_router.shape[-2]
    dt = _dt(x)
    shape = (G, T, k) if grouped else (T, k)
    if topk_idx is None:
        topk_idx = torch.empty(shape, dtype=torch.int32, device=x.device)
    if topk_w is None:
        topk_w = torch.empty(shape, dtype=torch.float32, device=x.device)
    args = (_dev(x, "x"), _dev(w_router, "w_router", x.dtype), _dev(bias, "bias", torch.float32),
            _dev(topk_idx, "topk_idx", torch.int32), _dev(topk_w, "topk_w", torch.float32),
            _stream(stream))
    if not grouped and gating == "renorm":
        _check(lib().foe_route(dt, T, d, E, k, *args), "foe_route")
    else:
        _check(lib().foe_route_ex(dt, G, T, d, E, k, _gating(gating), *args), "foe_route_ex")
    return topk_idx, topk_w


def permute(topk_idx, x, E, ws=None, stream=None, with_counts=True):
    """foe_permute: returns dict(counts, offsets, sorted_src, row_of, x_perm)."""
    T, k = topk_idx.shape
    d = x.shape[1]
    dt = _dt(x)
    dev = x.device
    R = T * k
    out = {
        "counts": torch.empty(E, dtype=torch.int32, device=dev) if with_counts else None,
        "offsets": torch.empty(E + 1, dtype=torch.int32, device=dev),
        "sorted_src": torch.empty(R, dtype=torch.int32, device=dev),
        "row_of": torch.empty(R, dtype=torch.int32, device=dev),
        "x_perm": torch.empty((R, d), dtype=x.dtype, device=dev),
    }
    need = workspace_bytes("permute", dt, 1, T, d, E, k, 0)
    ws = _workspace(ws, need, dev)
    rc = lib().foe_permute(dt, T, d, E, k, _dev(topk_idx, "topk_idx", torch.int32), _dev(x, "x"),
                           _dev(out["counts"], "counts"), _dev(out["offsets"], "offsets"),
                           _dev(out["sorted_src"], "sorted_src"), _dev(out["row_of"], "row_of"),
                           _dev(out["x_perm"], "x_perm"), _dev(ws, "ws"), ws.numel(),
                           _stream(stream))
    _check(rc, "foe_permute")
    return out


def expert_ffn(x_perm, offsets, w_gate, w_up, w_down, y_perm=None, ws=None, stream=None):
    """foe_expert_ffn: returns y_perm [rows,d]."""
    rows, d = x_perm.shape
    E, F, _ = w_gate.shape
    dt = _dt(x_perm)
    if y_perm is None:
        y_perm = torch.empty((rows, d), dtype=x_perm.dtype, device=x_perm.device)
    need = workspace_bytes("expert_ffn", dt, 1, rows, d, E, 1, F)
    ws = _workspace(ws, need, x_perm.device)
    rc = lib().foe_expert_ffn(dt, E, d, F, rows, _dev(x_perm, "x_perm"),
                              _dev(offsets, "offsets", torch.int32),
                              _dev(w_gate, "w_gate", x_perm.dtype), _dev(w_up, "w_up", x_perm.dtype),
                              _dev(w_down, "w_down", x_perm.dtype),
                              _dev(y_perm, "y_perm", x_perm.dtype), _dev(ws, "ws"), ws.numel(),
                              _stream(stream))
    _check(rc, "foe_expert_ffn")
    return y_perm


def combine(y_perm, row_of, topk_w, residual=None, out=None, stream=None):
    """foe_combine: returns out [T,d]."""
    T, k = topk_w.shape
    d = y_perm.shape[1]
    dt = _dt(y_perm)
    if out is None:
        out = torch.empty((T, d), dtype=y_perm.dtype, device=y_perm.device)
    rc = lib().foe_combine(dt, T, d, k, _dev(y_perm, "y_perm"), _dev(row_of, "row_of", torch.int32),
                           _dev(topk_w, "topk_w", torch.float32),
                           _dev(residual, "residual", y_perm.dtype), _dev(out, "out", y_perm.dtype),
                           _stream(stream))
    _check(rc, "foe_combine")
    return out


def reduce(partials, scale, residual=None, out=None, stream=None):
    """foe_reduce: out = scale * sum_h (residual + partials[h])."""
    C, T, d = partials.shape
    dt = _dt(partials)
    if out is None:
        out = torch.empty((T, d), dtype=partials.dtype, device=partials.device)
    rc = lib().foe_reduce(dt, C, T, d, _dev(partials, "partials"),
                          _dev(residual, "residual", partials.dtype), float(scale),
                          _dev(out, "out", partials.dtype), _stream(stream))
    _check(rc, "foe_reduce")
    return out


def cluster_block(x, w_router, bias, w_gate, w_up, w_down, k, reduce_scale=None, out=None,
                  ws=None, stream=None, gating="renorm"):
    """foe_cluster_block (foe_cluster_block_ex for a gating other than "renorm")
    for C clusters: weights stacked on a leading C axis."""
    T, d = x.shape
    C, E, F, _ = w_gate.shape
    dt = _dt(x)
    if reduce_scale is None:
        reduce_scale = 1.0 / C
    if out is None:
        out = torch.empty((T, d), dtype=x.dtype, device=x.device)
    need = workspace_bytes("cluster_block", dt, C, T, d, E, k, F)
    ws = _workspace(ws, need, x.device)
    args = (_dev(x, "x"), _dev(w_router, "w_router", x.dtype), _dev(bias, "bias", torch.float32),
            _dev(w_gate, "w_gate", x.dtype), _dev(w_up, "w_up", x.dtype),
            _dev(w_down, "w_down", x.dtype), float(reduce_scale), _dev(out, "out", x.dtype),
            _dev(ws, "ws"), ws.numel(), _stream(stream))
    if gating == "renorm":
        _check(lib().foe_cluster_block(dt, C, T, d, E, k, F, *args), "foe_cluster_block")
    else:
        _check(lib().foe_cluster_block_ex(dt, C, T, d, E, k, F, _gating(gating), *args),
               "foe_cluster_block_ex")
    return out


# bytes of the per-GPU scratch array of foe_cluster_block_noalloc
NOALLOC_SCRATCH_BYTES = 128 << 20


def cluster_block_noalloc(x, w_router, bias, w_gate, w_up, w_down, k, reduce_scale=None,
                          out=None, stream=None):
    """foe_cluster_block_noalloc: foe_cluster_block without a workspace (the
    library's per-GPU scratch array); weights stacked on a leading C axis."""
    T, d = x.shape
    C, E, F, _ = w_gate.shape
    if reduce_scale is None:
        reduce_scale = 1.0 / C
    if out is None:
        out = torch.empty((T, d), dtype=x.dtype, device=x.device)
    _check(lib().foe_cluster_block_noalloc(
        _dt(x), C, T, d, E, k, F, _dev(x, "x"), _dev(w_router, "w_router", x.dtype),
        _dev(bias, "bias", torch.float32), _dev(w_gate, "w_gate", x.dtype),
        _dev(w_up, "w_up", x.dtype), _dev(w_down, "w_down", x.dtype), float(reduce_scale),
        _dev(out, "out", x.dtype), _stream(stream)), "foe_cluster_block_noalloc")
    return out


def group_attention(x, w_qkv, w_o, nq, theta, scale=1.0, out=None, ws=None, stream=None):
    """foe_group_attention: x [H,S,d], w_qkv [H,(nq+2)*hd,d], w_o [d,H*nq*hd]
    (the groups' output projections side by side; bf16, hd = 96 or 128) ->
    r_full [S,d]."""
    H, S, d = x.shape
    hd = w_qkv.shape[1] // (nq + 2)
    if tuple(w_qkv.shape) != (H, (nq + 2) * hd, d) or tuple(w_o.shape) != (d, H * nq * hd):
        raise FoeError(FOE_ERR_INVALID, f"group_attention: w_qkv {tuple(w_qkv.shape)} / w_o "
                       f"{tuple(w_o.shape)} do not match x {tuple(x.shape)} with nq={nq}")
    if out is None:
        out = torch.empty((S, d), dtype=x.dtype, device=x.device)
    n = lib().foe_group_attention_workspace_bytes(H, S, d, nq, hd)
    if n == ctypes.c_size_t(-1).value:
        raise FoeError(FOE_ERR_INVALID, f"foe_group_attention_workspace_bytes: {last_error()}")
    ws = _workspace(ws, n, x.device)
    rc = lib().foe_group_attention(_dt(x), H, S, d, nq, hd, float(theta), float(scale),
                                   _dev(x, "x"), _dev(w_qkv, "w_qkv", x.dtype),
                                   _dev(w_o, "w_o", x.dtype), _dev(out, "r_full", x.dtype),
                                   _dev(ws, "ws"), ws.numel(), _stream(stream))
    _check(rc, "foe_group_attention")
    return out


# ---- the 8-bit key/value cache --------------------------------------------------

CACHE_PAGE = 64  # tokens per page


def cache_empty(n_pages, H, hd, device="cuda"):
    """A pool of pages: dict(k, v, kv_scale, mass), with zero masses and scales
    of the smallest value (the codes are not initialised)."""
    f8 = torch.float8_e4m3fn
    return {"k": torch.empty((n_pages, H, CACHE_PAGE, hd), dtype=f8, device=device),
            "v": torch.empty((n_pages, H, CACHE_PAGE // 16, hd, 16), dtype=f8, device=device),
            "kv_scale": torch.full((n_pages, H, 2), 2.0 ** -100, device=device),
            "mass": torch.zeros((n_pages, H, CACHE_PAGE), device=device)}


def _on(device, stream):
    """Context in which a call allocates and launches: the tensors' device, and
    `stream` as the current one, so that what the call allocates for itself belongs
    to the stream that uses it."""
    if device.type != "cuda":
        raise TypeError("GPU tensors are needed")
    if stream is None:
        return torch.cuda.device(device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    return torch.cuda.stream(stream)


def _stream_of(dev):
    """Handle of the current stream of device ``dev``."""
    return torch._C._cuda_getCurrentRawStream(dev)


def _elsewhere(t, stream):
    """Whether a call on ``t`` needs that context.  (A decode step's calls take a few
    microseconds on the GPU, so what they cost on the host counts.)"""
    return stream is not None or t.get_device() != torch.cuda.current_device()


def _arg(t, name, dtype, shape, dev):
    """Device pointer of a contiguous tensor of that dtype and shape on device ``dev``."""
    if (t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == dev):
        return t.data_ptr()
    if t.get_device() != dev:
        raise ValueError(f"tensors on cuda:{dev} and {t.device} ({name})")
    if t.shape != shape:
        raise FoeError(FOE_ERR_INVALID, f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    return _dev(t, name, dtype)  # raises


def _pool_args(k, v, kv_scale, n_pages, H, hd, dev):
    f8 = torch.float8_e4m3fn
    return (_arg(k, "k", f8, (n_pages, H, CACHE_PAGE, hd), dev),
            _arg(v, "v", f8, (n_pages, H, CACHE_PAGE // 16, hd, 16), dev),
            _arg(kv_scale, "kv_scale", torch.float32, (n_pages, H, 2), dev))


def _ws_arg(ws, nbytes, device, dev):
    """A workspace of nbytes() bytes, or the caller's (the library refuses one that is too
    small): (tensor, pointer, bytes)."""
    if ws is None:
        ws = torch.empty(max(nbytes(), 1), dtype=torch.uint8, device=device)
    return ws, _arg(ws, "ws", torch.uint8, ws.shape, dev), ws.numel()


def _size(n, name):
    if n == ctypes.c_size_t(-1).value:
        raise FoeError(FOE_ERR_INVALID, f"{name}: {last_error()}")
    return n


def cache_append(qkv, k, v, kv_scale, block_table, ctx_len, row_start, theta, scale=1.0, pos=None,
                 q=None, stream=None):
    """foe_cache_append: qkv [H,N,nq+2,hd] into the pages of block_table
    [B,max_blocks]; returns the rotated queries [H,N,nq,hd]."""
    if _elsewhere(qkv, stream):
        with _on(qkv.device, stream):
            return cache_append(qkv, k, v, kv_scale, block_table, ctx_len, row_start, theta, scale,
                                pos, q)
    n_pages, H, _, hd = k.shape
    N, nq = qkv.shape[1], qkv.shape[2] - 2
    B, max_blocks = block_table.shape
    dev, i32, dt = qkv.get_device(), torch.int32, _dt(qkv)
    if q is None:
        q = torch.empty((H, N, nq, hd), dtype=qkv.dtype, device=qkv.device)
    rc = lib().foe_cache_append(
        dt, H, B, N, nq, hd, n_pages, max_blocks, theta, scale,
        _arg(qkv, "qkv", qkv.dtype, (H, N, nq + 2, hd), dev),
        _arg(row_start, "row_start", i32, (B + 1,), dev), _arg(ctx_len, "ctx_len", i32, (B,), dev),
        None if pos is None else _arg(pos, "pos", i32, (B,), dev),
        _arg(block_table, "block_table", i32, (B, max_blocks), dev),
        _arg(q, "q", qkv.dtype, (H, N, nq, hd), dev),
        *_pool_args(k, v, kv_scale, n_pages, H, hd, dev), _stream_of(dev))
    _check(rc, "foe_cache_append")
    return q


def cache_attention_workspace_bytes(q, block_table, max_rows, with_mass=False):
    """Workspace bytes of cache_attention for these tensors."""
    H, N, nq, hd = q.shape
    B, max_blocks = block_table.shape
    return _size(lib().foe_cache_attention_workspace_bytes(H, B, N, nq, hd, max_blocks, max_rows,
                                                           1 if with_mass else 0),
                 "foe_cache_attention_workspace_bytes")


def cache_attention(q, k, v, kv_scale, block_table, ctx_len, row_start, max_rows, mass_in=None,
                    mass_out=None, out=None, ws=None, stream=None):
    """foe_cache_attention: q [H,N,nq,hd] over the pages of block_table; returns
    out [N,H,nq,hd]."""
    if _elsewhere(q, stream):
        with _on(q.device, stream):
            return cache_attention(q, k, v, kv_scale, block_table, ctx_len, row_start, max_rows,
                                   mass_in, mass_out, out, ws)
    n_pages, H, _, hd = k.shape
    N, nq = q.shape[1], q.shape[2]
    B, max_blocks = block_table.shape
    dev, i32, f32, dt = q.get_device(), torch.int32, torch.float32, _dt(q)
    mshape = (n_pages, H, CACHE_PAGE)
    if out is None:
        out = torch.empty((N, H, nq, hd), dtype=q.dtype, device=q.device)
    ws, ws_ptr, ws_bytes = _ws_arg(
        ws, lambda: cache_attention_workspace_bytes(q, block_table, max_rows,
                                                    mass_out is not None), q.device, dev)
    rc = lib().foe_cache_attention(
        dt, H, B, N, nq, hd, n_pages, max_blocks, max_rows,
        _arg(q, "q", q.dtype, (H, N, nq, hd), dev),
        _arg(row_start, "row_start", i32, (B + 1,), dev), _arg(ctx_len, "ctx_len", i32, (B,), dev),
        _arg(block_table, "block_table", i32, (B, max_blocks), dev),
        *_pool_args(k, v, kv_scale, n_pages, H, hd, dev),
        None if mass_in is None else _arg(mass_in, "mass_in", f32, mshape, dev),
        None if mass_out is None else _arg(mass_out, "mass_out", f32, mshape, dev),
        _arg(out, "out", q.dtype, (N, H, nq, hd), dev), ws_ptr, ws_bytes, _stream_of(dev))
    _check(rc, "foe_cache_attention")
    return out


def cache_evict_workspace_bytes(block_table, H):
    """Workspace bytes of cache_evict for a table and H groups."""
    B, max_blocks = block_table.shape
    return _size(lib().foe_cache_evict_workspace_bytes(H, B, max_blocks),
                 "foe_cache_evict_workspace_bytes")


def cache_evict(k, v, kv_scale, mass, block_table, length, keep, recent, dst_table, kept=None,
                new_len=None, ws=None, stream=None):
    """foe_cache_evict: returns (kept [B,H,keep], new_len [B])."""
    if _elsewhere(k, stream):
        with _on(k.device, stream):
            return cache_evict(k, v, kv_scale, mass, block_table, length, keep, recent, dst_table,
                               kept, new_len, ws)
    n_pages, H, _, hd = k.shape
    B, max_blocks = block_table.shape
    dst_blocks = dst_table.shape[-1]
    dev, i32 = k.get_device(), torch.int32
    if kept is None:
        kept = torch.empty((B, H, max(keep, 0)), dtype=i32, device=k.device)
    if new_len is None:
        new_len = torch.empty((B,), dtype=i32, device=k.device)
    ws, ws_ptr, ws_bytes = _ws_arg(ws, lambda: cache_evict_workspace_bytes(block_table, H),
                                   k.device, dev)
    rc = lib().foe_cache_evict(
        H, B, hd, n_pages, max_blocks, keep, recent, _arg(length, "length", i32, (B,), dev),
        _arg(block_table, "block_table", i32, (B, max_blocks), dev),
        _arg(dst_table, "dst_table", i32, (B, dst_blocks), dev), dst_blocks,
        *_pool_args(k, v, kv_scale, n_pages, H, hd, dev),
        _arg(mass, "mass", torch.float32, (n_pages, H, CACHE_PAGE), dev),
        _arg(kept, "kept", i32, (B, H, keep), dev), _arg(new_len, "new_len", i32, (B,), dev),
        ws_ptr, ws_bytes, _stream_of(dev))
    _check(rc, "foe_cache_evict")
    return kept, new_len


# ---- kernel timing -------------------------------------------------------------

def profile_enable(on=True):
    _check(lib().foe_profile_enable(1 if on else 0), "foe_profile_enable")


def profile_reset():
    _check(lib().foe_profile_reset(), "foe_profile_reset")


def profile_kernel(name):
    """(launches, total_ms) recorded for kernel ``name``."""
    n = ctypes.c_int(0)
    ms = ctypes.c_double(0.0)
    _check(lib().foe_profile_kernel(name.encode(), ctypes.byref(n), ctypes.byref(ms)),
           "foe_profile_kernel")
    return n.value, ms.value


def profile_names():
    need = lib().foe_profile_names(None, 0)
    buf = ctypes.create_string_buffer(need)
    lib().foe_profile_names(buf, need)
    s = buf.value.decode()
    return [t for t in s.split(",") if t]
