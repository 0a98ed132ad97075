"""ctypes binding of the 8-bit paged cache's operators (include/m2r2_kv8.h).

Argument checks and marshalling only, as in ``binding``.  Tensors of one call
are on one GPU; the call runs on that GPU's current stream unless one is
given, whichever device is current.
"""
from __future__ import annotations

import ctypes
import struct
from ctypes import POINTER, c_char_p, c_float, c_int32, c_int64, c_size_t, c_void_p
from typing import Optional

from .binding import BF16, F32, _check, lib

# include/m2r2_kv8.h
KV8_EXPORTS = ("m2r2_kv8_append", "m2r2_kv8_workspace_size", "m2r2_kv8_attention")
ERR_BLOCK, ERR_ROPE, ERR_ROWS = 2, 8, 32


class _Pages(ctypes.Structure):
    _fields_ = [("k_pages", c_void_p), ("v_pages", c_void_p), ("k_scales", c_void_p), ("v_scales", c_void_p),
                ("block_table_d", c_void_p), ("num_blocks", c_int32), ("block_size", c_int32),
                ("max_blocks_per_seq", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32)]


class _Rows(ctypes.Structure):
    _fields_ = [("n_seqs", c_int32), ("n_rows", c_int32), ("row_start_d", c_void_p), ("positions_d", c_void_p),
                ("dtype", c_int32), ("k", c_void_p), ("v", c_void_p), ("k_row", c_int64), ("k_head", c_int64),
                ("v_row", c_int64), ("v_head", c_int64), ("rope_d", c_void_p), ("rope_len", c_int32),
                ("n_heads", c_int32), ("q", c_void_p), ("q_out", c_void_p), ("q_row", c_int64), ("q_head", c_int64),
                ("qo_row", c_int64), ("qo_head", c_int64), ("err_d", c_void_p)]


class _Query(ctypes.Structure):
    _fields_ = [("n_seqs", c_int32), ("n_rows", c_int32), ("row_start_d", c_void_p), ("lens_d", c_void_p),
                ("visible_d", c_void_p), ("dtype", c_int32), ("n_heads", c_int32), ("q", c_void_p),
                ("q_row", c_int64), ("q_head", c_int64), ("own_d", c_void_p), ("own_k", c_void_p), ("own_v", c_void_p),
                ("n_own", c_int32), ("ok_row", c_int64), ("ok_head", c_int64), ("ov_row", c_int64),
                ("ov_head", c_int64), ("scale", c_float), ("out", c_void_p), ("out_row", c_int64),
                ("out_head", c_int64), ("err_d", c_void_p)]


# The last two as struct formats (native alignment): filling one takes a quarter of
# the time of building the ctypes structure.
_ROWS = struct.Struct("@iiPPiPPqqqqPiiPPqqqqP")
_QUERY = struct.Struct("@iiPPPiiPqqPPPiqqqqfPqqP")

_fns = None
_packed_fns = None


def _packed():
    """(append, attention) that take descriptions as bytes."""
    global _packed_fns
    if _packed_fns is None:
        L = lib()
        append, attention = L["m2r2_kv8_append"], L["m2r2_kv8_attention"]   # (function objects of their own)
        append.argtypes = [c_char_p, c_char_p, c_void_p]
        attention.argtypes = [c_char_p, c_char_p, c_void_p, c_size_t, c_void_p]
        append.restype = attention.restype = c_int32
        _packed_fns = (append, attention)
    return _packed_fns


def _lib():
    """(append, workspace size, attention) with their signatures set."""
    global _fns
    if _fns is None:
        L = lib()
        L.m2r2_kv8_append.argtypes = [POINTER(_Pages), POINTER(_Rows), c_void_p]
        L.m2r2_kv8_workspace_size.argtypes = [POINTER(_Pages), c_int32, c_int32, c_int32, POINTER(c_size_t)]
        L.m2r2_kv8_attention.argtypes = [POINTER(_Pages), POINTER(_Query), c_void_p, c_size_t, c_void_p]
        for f in KV8_EXPORTS:
            getattr(L, f).restype = c_int32
        _fns = (L.m2r2_kv8_append, L.m2r2_kv8_workspace_size, L.m2r2_kv8_attention)
    return _fns


class KV8Pages:
    """One layer of an 8-bit paged cache: ``k_pages``/``v_pages``
    ``[num_blocks][n_kv_heads][block_size][head_dim]`` float8_e4m3fn codes,
    ``k_scales``/``v_scales`` ``[num_blocks][n_kv_heads]`` float32 powers of two, and
    the block table ``[n_seqs][max_blocks_per_seq]`` int32.  The tensors are the
    caller's; a cached value is code * scale."""

    def __init__(self, k_pages, v_pages, k_scales, v_scales, block_table):
        import torch
        if k_pages.dim() != 4 or k_pages.dtype != torch.float8_e4m3fn or not k_pages.is_contiguous():
            raise ValueError("k_pages: a contiguous float8_e4m3fn tensor [blocks][heads][block size][head dim]")
        for name, t, like in (("v_pages", v_pages, k_pages), ("v_scales", v_scales, k_scales)):
            if t.shape != like.shape or t.dtype != like.dtype or not t.is_contiguous():
                raise ValueError(f"{name}: contiguous, of the keys' shape and type")
        if k_scales.shape != k_pages.shape[:2] or k_scales.dtype != torch.float32 or not k_scales.is_contiguous():
            raise ValueError("k_scales: a contiguous float32 tensor [blocks][heads]")
        if block_table.dim() != 2 or block_table.dtype != torch.int32 or not block_table.is_contiguous():
            raise ValueError("block_table: a contiguous int32 tensor [sequences][blocks]")
        self.device = k_pages.device
        if any(t.device != self.device for t in (v_pages, k_scales, v_scales, block_table)):
            raise ValueError("the cache's tensors are on different devices")
        self.k_pages, self.v_pages, self.k_scales, self.v_scales = k_pages, v_pages, k_scales, v_scales
        self.block_table = block_table
        nb, H, bs, hd = k_pages.shape
        self.gpu = k_pages.get_device()   # (-1: not on one)
        self.n_seqs, self.n_kv_heads, self.head_dim = block_table.shape[0], H, hd
        self._desc = _Pages(k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(),
                            block_table.data_ptr(), nb, bs, block_table.shape[1], H, hd)
        self._bytes = bytes(self._desc)


_torch = None


def _t():
    """torch, imported on first use as in ``binding``."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


# A decoding step makes these calls for every layer, and its kernels take a few
# microseconds each: the checks below look at every tensor once.

def _int32s(t, n: int, name: str, gpu: int) -> int:
    """Pointer to a vector of at least n int32 on the GPU (None: 0)."""
    if t is None:
        return 0
    if t.dim() != 1 or t.numel() < n or t.dtype is not _t().int32 or not t.is_contiguous() or t.get_device() != gpu:
        raise ValueError(f"{name}: a contiguous int32 vector of at least {n} entries on GPU {gpu}, "
                         f"not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _rows(t, name: str, shape: tuple, dtype, gpu: int):
    """(pointer, row stride, head stride) of a [n][heads][hd] tensor."""
    if t.shape == shape and t.dtype is dtype and t.get_device() == gpu:
        row, head, dim = t.stride()
        if dim == 1:
            return t.data_ptr(), row, head
    raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, strides {tuple(t.stride())} on {t.device}; "
                     f"expected {dtype} {shape} with adjacent dims on GPU {gpu}")


def _dtype(t, name: str):
    torch = _t()
    dt = t.dtype
    if dt is torch.bfloat16:
        return BF16, dt
    if dt is torch.float32:
        return F32, dt
    raise ValueError(f"{name}: {dt} (bfloat16 or float32)")


def _call(fn, where: str, kv, stream, *args) -> None:
    """fn(*args, stream) with the cache's GPU current."""
    gpu, torch = kv.gpu, _t()
    if gpu < 0:
        raise ValueError(f"{where}: tensors on {kv.device}")
    if stream is not None:
        s = stream.cuda_stream
    else:   # (the handle without a Stream object around it, which takes a microsecond)
        s = torch._C._cuda_getCurrentRawStream(gpu)
    if torch._C._cuda_getDevice() == gpu:
        st = fn(*args, s)
    else:
        with torch.cuda.device(gpu):
            st = fn(*args, s)
    if st:
        _check(st, where)


def kv8_append(kv: KV8Pages, k, v, row_start, positions, *, rope=None, q=None, q_out=None, errors=None,
               stream=None) -> None:
    """Append rows ``k``/``v`` [rows][n_kv_heads][head_dim] to the cache: rows
    row_start[s] .. row_start[s+1]-1 are sequence s's, from ``positions[s]`` on.
    ``rope`` [length][head_dim/2][2] float32 (cos, sin) turns the keys (and the
    queries ``q`` [rows][heads][head_dim] into ``q_out``, which may be ``q``).
    ``errors``: an int32 tensor into which the kernels or error bits."""
    n, H, hd, ns, gpu = len(k), kv.n_kv_heads, kv.head_dim, kv.n_seqs, kv.gpu
    code, dt = _dtype(k, "k")
    shape = (n, H, hd)
    kp, k_row, k_head = _rows(k, "k", shape, dt, gpu)
    vp, v_row, v_head = _rows(v, "v", shape, dt, gpu)
    heads, qp, q_row, q_head, op, o_row, o_head = 0, 0, 0, 0, 0, 0, 0
    if q is not None and q_out is not None:
        heads = q.shape[1] if q.dim() == 3 else 0
        shape = (n, heads, hd)
        qp, q_row, q_head = _rows(q, "q", shape, dt, gpu)
        op, o_row, o_head = (qp, q_row, q_head) if q_out is q else _rows(q_out, "q_out", shape, dt, gpu)
    elif q is not None or q_out is not None:
        raise ValueError("q and q_out come together")
    rp, rlen = 0, 0
    if rope is not None:
        rlen = len(rope)
        if (rope.shape != (rlen, hd // 2, 2) or rope.dtype is not _t().float32 or not rope.is_contiguous()
                or rope.get_device() != gpu):
            raise ValueError("rope: a contiguous float32 tensor [length][head_dim/2][2] on the cache's GPU")
        rp = rope.data_ptr()
    r = _ROWS.pack(ns, n, _int32s(row_start, ns + 1, "row_start", gpu), _int32s(positions, ns, "positions", gpu), code,
                   kp, vp, k_row, k_head, v_row, v_head, rp, rlen, heads, qp, op, q_row, q_head, o_row, o_head,
                   _int32s(errors, 1, "errors", gpu))
    _call(_packed()[0], "m2r2_kv8_append", kv, stream, kv._bytes, r)


def kv8_workspace(kv: KV8Pages, q):
    """A zeroed workspace for ``kv8_attention`` calls of queries shaped like
    ``q``, or smaller, over this cache.  Calls that may overlap need one each."""
    import torch
    n = c_size_t(0)
    _check(_lib()[1](kv._desc, kv.n_seqs, q.shape[0], q.shape[1], n), "m2r2_kv8_workspace_size")
    return torch.zeros(n.value, dtype=torch.uint8, device=kv.device)


def kv8_attention(kv: KV8Pages, q, row_start, lens, out, workspace, *, visible=None, own=None, own_k=None, own_v=None,
                  scale: Optional[float] = None, errors=None, stream=None) -> None:
    """``out`` = softmax(scale * q K^T) V of rows ``q`` [rows][heads][head_dim]
    over the first ``lens[s]`` positions of their sequences: row r sees
    min(visible[r], lens[s]) of them (None: causal, the sequence's last row sees
    all) and, where own[r] >= 0, the key and value own_k/own_v[own[r]] beside
    them.  A row that sees nothing is zero."""
    if q.dim() != 3:
        raise ValueError(f"q: {tuple(q.shape)}; expected [rows][heads][head_dim]")
    n, heads, H, hd, ns, gpu = q.shape[0], q.shape[1], kv.n_kv_heads, kv.head_dim, kv.n_seqs, kv.gpu
    if scale is not None and not scale > 0:
        raise ValueError(f"scale {scale}")
    code, dt = _dtype(q, "q")
    shape = (n, heads, hd)
    qp, q_row, q_head = _rows(q, "q", shape, dt, gpu)
    op, o_row, o_head = _rows(out, "out", shape, dt, gpu)
    n_own, wp, kp, k_row, k_head, vp, v_row, v_head = 0, 0, 0, 0, 0, 0, 0, 0
    if own is not None and own_k is not None and own_v is not None:
        n_own = len(own_k)
        shape = (n_own, H, hd)
        kp, k_row, k_head = _rows(own_k, "own_k", shape, dt, gpu)
        vp, v_row, v_head = _rows(own_v, "own_v", shape, dt, gpu)
        wp = _int32s(own, n, "own", gpu) if n_own else 0
    elif own is not None or own_k is not None or own_v is not None:
        raise ValueError("own, own_k and own_v come together")
    if workspace.get_device() != gpu or not workspace.is_contiguous():
        raise ValueError(f"workspace: a contiguous tensor on GPU {gpu}")
    a = _QUERY.pack(ns, n, _int32s(row_start, ns + 1, "row_start", gpu), _int32s(lens, ns, "lens", gpu),
                    _int32s(visible, n, "visible", gpu), code, heads, qp, q_row, q_head, wp, kp, vp, n_own, k_row, k_head,
                    v_row, v_head, 0.0 if scale is None else scale, op, o_row, o_head, _int32s(errors, 1, "errors", gpu))
    _call(_packed()[1], "m2r2_kv8_attention", kv, stream, kv._bytes, a, workspace.data_ptr(), workspace.nbytes)
