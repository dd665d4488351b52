"""Thin ctypes binding of libdecomoe_block.so (C ABI in include/decomoe_block.h):
the attention half of a decoder block over a paged cache.

Like ``abi``: argument marshalling only.  Functions carry the C names; arrays
are contiguous torch tensors on the current GPU, sizes are taken from them and
checked against each other, and the stream defaults to torch's current stream.
A non-zero status raises ``abi.MoeError``.  There is no fallback: without the
built library every call raises.

8-bit rows are a ``torch.float8_e4m3fn`` (or uint8) tensor and a
``torch.float8_e8m0fnu`` (or uint8) tensor of one scale for every 32 values;
4-bit weights are uint8 codes, two to a byte, with the same scales.
"""

from __future__ import annotations

import ctypes
import os

import torch

from .abi import MOE_BF16, MOE_F32, _check

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdecomoe_block.so")

BLK_MX8 = 2
BLOCK = 32  # values of one scale

EXPORTS = ("blk_rms_norm", "blk_kv_extend", "blk_qkv_cache", "blk_attn_workspace_size", "blk_attn_decode",
           "blk_linear_w4", "blk_quantize_w4")

_lib = None
_P, _I, _D, _S = ctypes.c_void_p, ctypes.c_int, ctypes.c_double, ctypes.c_size_t


def load() -> ctypes.CDLL:
    """Load the in-tree library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_38823_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    sig = {
        "blk_rms_norm": (_I, [_P, _I, _P, _P, _I, _I, _D, _P, _P, _P, _P, _P]),
        "blk_kv_extend": (_I, [_P, _P, _I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
        "blk_qkv_cache": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _D, _P, _P, _I, _P, _I, _I, _I, _P, _P, _P, _P, _P,
                               _P]),
        "blk_attn_workspace_size": (_S, [_I, _I, _I, _I, _I]),
        "blk_attn_decode": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _P, _I, _I, _I, _P, _I, _P, _D, _P, _P, _S, _P]),
        "blk_linear_w4": (_I, [_P, _I, _P, _I, _I, _P, _P, _I, _P, _I, _P]),
        "blk_quantize_w4": (_I, [_P, _I, _I, _I, _P, _P, _P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    _lib = lib
    return lib


_F32, _I32 = (torch.float32,), (torch.int32,)
_E4M3 = (torch.float8_e4m3fn, torch.uint8)
_E8M0 = (getattr(torch, "float8_e8m0fnu", torch.uint8), torch.uint8)
_U8 = (torch.uint8,)
_ROWS = {torch.bfloat16: MOE_BF16, torch.float32: MOE_F32}
# the current device and its current stream's handle, without Python objects
# in between (calls of small steps are bound by the host)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, dev):
    if stream is None:
        return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _wrong(name, t, dtypes, want, dev):
    """Why an array is not taken."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: device arrays are passed as torch tensors")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} is {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    if t.get_device() != dev:  # the library launches on the current device
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{dev}")
    if not t.is_contiguous():
        raise ValueError(f"{name} is not contiguous")
    raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {want}")


def _arr(name, t, dtypes, shape, dev):
    """The address of an array of one of the dtypes and of this shape (None: NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.shape != shape or t.get_device() != dev \
            or not t.is_contiguous():
        _wrong(name, t, dtypes, shape, dev)
    return t.data_ptr()


def _vec(name, t, dtypes, n, dev):
    """The address of an array of n values (None: NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.numel() != n or t.get_device() != dev \
            or not t.is_contiguous():
        _wrong(name, t, dtypes, f"{n} values", dev)
    return t.data_ptr()


def _dt(name, t):
    dt = _ROWS.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name} is {t.dtype}, expected {' or '.join(map(str, _ROWS))}")
    return dt


def _cache(rows, k_cache, v_cache, k_scale, v_scale, dev):
    """(cache_dtype, addresses of the cache's four arrays) for rows of a dtype."""
    shape = k_cache.shape
    if len(shape) != 4:
        raise ValueError("the cache is [n_pages, n_kv, page_size, D]")
    mx = k_cache.dtype in _E4M3
    kinds = (k_cache.dtype,) if mx else (rows.dtype,)
    scales = (*shape[:3], shape[3] // BLOCK)
    return (BLK_MX8 if mx else _dt("rows", rows), _arr("k_cache", k_cache, kinds, shape, dev),
            _arr("v_cache", v_cache, kinds, shape, dev), _arr("k_scale", k_scale, _E8M0, scales, dev),
            _arr("v_scale", v_scale, _E8M0, scales, dev))


def blk_rms_norm(x, weight, eps, residual=None, h_out=None, y=None, q=None, q_scale=None, stream=None):
    """h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight: h_out, y (x's
    dtype) and (q, q_scale), y as 8-bit rows; h_out and y may be x or residual."""
    shape, dev, dt = x.shape, _device(), _dt("x", x)
    T, d = shape
    same = (x.dtype,)
    st = load().blk_rms_norm(
        _arr("x", x, same, shape, dev), dt, _arr("residual", residual, same, shape, dev),
        _vec("weight", weight, _F32, d, dev), T, d, eps, _arr("h_out", h_out, same, shape, dev),
        _arr("y", y, same, shape, dev), _arr("q", q, _E4M3, shape, dev),
        _arr("q_scale", q_scale, _E8M0, (T, -(-d // BLOCK)), dev), _stream(stream, dev))
    if st:
        _check("blk_rms_norm", st)


def blk_kv_extend(len_in, add, n_free_in, block_table, free_pages, page_size, len_out, n_free_out, row_offsets,
                  slot_map, positions, accepted, status, stream=None):
    """Page tables and slot maps of a step's new tokens (add < 0: the sequence
    is finished and gives its pages back); block_table and free_pages are
    updated, len_out may be len_in and n_free_out n_free_in."""
    (n_seq, max_pages), n_pages, rows, dev = block_table.shape, free_pages.numel(), slot_map.numel(), _device()
    st = load().blk_kv_extend(
        _vec("len_in", len_in, _I32, n_seq, dev), _vec("add", add, _I32, n_seq, dev), n_seq, page_size, max_pages,
        n_pages, rows, _vec("n_free_in", n_free_in, _I32, 1, dev),
        _arr("block_table", block_table, _I32, block_table.shape, dev),
        _vec("free_pages", free_pages, _I32, n_pages, dev), _vec("len_out", len_out, _I32, n_seq, dev),
        _vec("n_free_out", n_free_out, _I32, 1, dev), _vec("row_offsets", row_offsets, _I32, n_seq + 1, dev),
        _vec("slot_map", slot_map, _I32, rows, dev), _vec("positions", positions, _I32, rows, dev),
        _vec("accepted", accepted, _I32, n_seq, dev), _vec("status", status, _I32, 4, dev), _stream(stream, dev))
    if st:
        _check("blk_kv_extend", st)


def blk_qkv_cache(qkv, n_q, slot_map, k_cache, v_cache, q_out, positions=None, inv_freq=None, q_norm=None,
                  k_norm=None, eps=1e-6, k_scale=None, v_scale=None, stream=None):
    """qkv [T, (n_q + 2 n_kv) * D]: norm and rotation (inv_freq [rot / 2]) of
    the query and key heads; q_out [T, n_q, D], keys and values into the cache
    at slot_map."""
    dev, dt = _device(), _dt("qkv", qkv)
    kind, k, v, ks, vs = _cache(qkv, k_cache, v_cache, k_scale, v_scale, dev)
    n_pages, n_kv, page, D = k_cache.shape
    T, same = qkv.shape[0], (qkv.dtype,)
    rot = 2 * inv_freq.numel() if inv_freq is not None else 0
    st = load().blk_qkv_cache(
        _vec("qkv", qkv, same, T * (n_q + 2 * n_kv) * D, dev), dt, T, n_q, n_kv, D,
        _vec("q_norm", q_norm, _F32, D, dev), _vec("k_norm", k_norm, _F32, D, dev), eps,
        _vec("positions", positions, _I32, T, dev) if rot else None, _vec("inv_freq", inv_freq, _F32, rot // 2, dev), rot,
        _vec("slot_map", slot_map, _I32, T, dev), kind, n_pages, page, _arr("q_out", q_out, same, (T, n_q, D), dev), k, v,
        ks, vs, _stream(stream, dev))
    if st:
        _check("blk_qkv_cache", st)


def blk_attn_workspace_size(n_seq: int, n_q: int, n_kv: int, D: int, max_keys: int) -> int:
    return int(load().blk_attn_workspace_size(n_seq, n_q, n_kv, D, max_keys))


def blk_attn_decode(q, k_cache, v_cache, block_table, lens, scale, out, ws, k_scale=None, v_scale=None,
                    stream=None):
    """q [n_seq, n_q, D]: attention of one new token of each sequence over its
    lens[s] keys in the pages block_table[s]."""
    dev, dt, shape = _device(), _dt("q", q), q.shape
    kind, k, v, ks, vs = _cache(q, k_cache, v_cache, k_scale, v_scale, dev)
    n_pages, n_kv, page, D = k_cache.shape
    n_seq, n_q, last = shape
    if last != D:
        raise ValueError(f"q has heads of {last}, the cache of {D}")
    width, same = block_table.shape[-1], (q.dtype,)
    if ws is not None and (ws.get_device() != dev or not ws.is_contiguous()):
        raise ValueError("ws is contiguous memory of the current device")
    st = load().blk_attn_decode(
        _arr("q", q, same, shape, dev), dt, n_seq, n_q, n_kv, D, k, v, ks, vs, kind, n_pages, page,
        _arr("block_table", block_table, _I32, (n_seq, width), dev), width, _vec("lens", lens, _I32, n_seq, dev), scale,
        _arr("out", out, same, shape, dev), ws.data_ptr() if ws is not None else None,
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream, dev))
    if st:
        _check("blk_attn_decode", st)


def blk_linear_w4(x, codes, scales, y, x_scale=None, stream=None):
    """y [T, n] = x [T, k] (bf16, float32, or 8-bit rows with x_scale) times
    the transposed 4-bit weights codes [n, k / 2], scales [n, k / 32]."""
    (T, k), n, dev = x.shape, codes.shape[0], _device()
    mx = x.dtype in _E4M3
    st = load().blk_linear_w4(
        _arr("x", x, (x.dtype,), x.shape, dev), BLK_MX8 if mx else _dt("x", x),
        _arr("x_scale", x_scale, _E8M0, (T, k // BLOCK), dev), T, k, _arr("codes", codes, _U8, (n, k // 2), dev),
        _arr("scales", scales, _E8M0, (n, k // BLOCK), dev), n, _arr("y", y, (y.dtype,), (T, n), dev), _dt("y", y),
        _stream(stream, dev))
    if st:
        _check("blk_linear_w4", st)


def blk_quantize_w4(w, codes, scales, stream=None):
    """w [n, k] (bf16 or float32) -> codes [n, k / 2], scales [n, k / 32]."""
    (n, k), dev = w.shape, _device()
    _check("blk_quantize_w4", load().blk_quantize_w4(
        _arr("w", w, (w.dtype,), w.shape, dev), _dt("w", w), n, k, _arr("codes", codes, _U8, (n, k // 2), dev),
        _arr("scales", scales, _E8M0, (n, k // BLOCK), dev), _stream(stream, dev)))


__all__ = ["MOE_BF16", "MOE_F32", "BLK_MX8", "load", *EXPORTS]
