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

from .abi import MOE_BF16, MOE_F32, _check, _dt, _f32, _i32, _p, _stream

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


_E8M0 = getattr(torch, "float8_e8m0fnu", torch.uint8)
_BYTES = {"e4m3": (torch.float8_e4m3fn, torch.uint8), "e8m0": (_E8M0, torch.uint8), "codes": (torch.uint8,)}


def _bytes(t, kind):
    if t is not None and t.dtype not in _BYTES[kind]:
        raise TypeError(f"expected a tensor of {kind} bytes, got {t.dtype}")
    return _p(t)


def _shape(name, t, *want):
    if t is not None and tuple(t.shape) != want:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {want}")


def _size(name, t, want):
    if t is not None and t.numel() != want:
        raise ValueError(f"{name} holds {t.numel()} values, expected {want}")


def _like(name, t, ref):
    if t is not None and t.dtype != ref.dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {ref.dtype}")


def _here(*tensors):
    """The library launches on the current device: every array has to be there."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.is_cuda and t.device.index != dev:
            raise ValueError(f"an array is on {t.device}, the current device is cuda:{dev}")


def _cache_dt(cache, rows):
    """cache_dtype of a cache that goes with rows of a dtype."""
    if cache.dtype in _BYTES["e4m3"]:
        return BLK_MX8
    _like("the cache", cache, rows)
    return _dt(cache)


def _cache_checks(k_cache, v_cache, k_scale, v_scale):
    if k_cache.dim() != 4:
        raise ValueError("the cache is [n_pages, n_kv, page_size, D]")
    _shape("v_cache", v_cache, *k_cache.shape)
    if v_cache.dtype != k_cache.dtype:
        raise TypeError("k_cache and v_cache differ in dtype")
    n_pages, n_kv, page, D = k_cache.shape
    for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
        _shape(name, t, n_pages, n_kv, page, D // BLOCK)


def blk_rms_norm(x, weight, eps, residual=None, h_out=None, y=None, q=None, q_scale=None, stream=None):
    """h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight: h_out, y (x's
    dtype) and (q, q_scale), y as 8-bit rows; h_out and y may be x or residual."""
    T, d = x.shape
    for name, t in (("residual", residual), ("h_out", h_out), ("y", y)):
        _shape(name, t, T, d)
        _like(name, t, x)
    _shape("q", q, T, d)
    _shape("q_scale", q_scale, T, -(-d // BLOCK))
    _size("weight", weight, d)
    _here(x, weight, residual, h_out, y, q, q_scale)
    _check("blk_rms_norm", load().blk_rms_norm(
        _p(x), _dt(x), _p(residual), _f32(weight), T, d, float(eps), _p(h_out), _p(y), _bytes(q, "e4m3"),
        _bytes(q_scale, "e8m0"), _stream(stream)))


def blk_kv_extend(len_in, add, n_free_in, block_table, free_pages, page_size, len_out, n_free_out, row_offsets,
                  slot_map, positions, accepted, status, stream=None):
    """Page tables and slot maps of a step's new tokens (add < 0: the sequence
    is finished and gives its pages back); block_table and free_pages are
    updated, len_out may be len_in and n_free_out n_free_in."""
    n_seq, max_pages = block_table.shape
    for name, t, want in (("len_in", len_in, n_seq), ("add", add, n_seq), ("n_free_in", n_free_in, 1),
                          ("len_out", len_out, n_seq), ("n_free_out", n_free_out, 1),
                          ("row_offsets", row_offsets, n_seq + 1), ("positions", positions, slot_map.numel()),
                          ("accepted", accepted, n_seq), ("status", status, 4)):
        _size(name, t, want)
    _here(len_in, add, n_free_in, block_table, free_pages, len_out, n_free_out, row_offsets, slot_map, positions,
          accepted, status)
    _check("blk_kv_extend", load().blk_kv_extend(
        _i32(len_in), _i32(add), n_seq, int(page_size), max_pages, free_pages.numel(), slot_map.numel(),
        _i32(n_free_in), _i32(block_table), _i32(free_pages), _i32(len_out), _i32(n_free_out), _i32(row_offsets),
        _i32(slot_map), _i32(positions), _i32(accepted), _i32(status), _stream(stream)))


def blk_qkv_cache(qkv, n_q, slot_map, k_cache, v_cache, q_out, positions=None, inv_freq=None, q_norm=None,
                  k_norm=None, eps=1e-6, k_scale=None, v_scale=None, stream=None):
    """qkv [T, (n_q + 2 n_kv) * D]: norm and rotation (inv_freq [rot / 2]) of
    the query and key heads; q_out [T, n_q, D], keys and values into the cache
    at slot_map."""
    _cache_checks(k_cache, v_cache, k_scale, v_scale)
    n_pages, n_kv, page, D = k_cache.shape
    T = qkv.shape[0]
    _size("qkv", qkv, T * (n_q + 2 * n_kv) * D)
    _shape("q_out", q_out, T, n_q, D)
    _like("q_out", q_out, qkv)
    for name, t, want in (("slot_map", slot_map, T), ("positions", positions, T), ("q_norm", q_norm, D),
                          ("k_norm", k_norm, D)):
        _size(name, t, want)
    rot = 2 * inv_freq.numel() if inv_freq is not None else 0
    _here(qkv, slot_map, k_cache, v_cache, q_out, positions, inv_freq, q_norm, k_norm, k_scale, v_scale)
    _check("blk_qkv_cache", load().blk_qkv_cache(
        _p(qkv), _dt(qkv), T, int(n_q), n_kv, D, _f32(q_norm), _f32(k_norm), float(eps),
        _i32(positions) if rot else None, _f32(inv_freq), rot, _i32(slot_map), _cache_dt(k_cache, qkv), n_pages, page,
        _p(q_out), _p(k_cache), _p(v_cache), _bytes(k_scale, "e8m0"), _bytes(v_scale, "e8m0"), _stream(stream)))


def blk_attn_workspace_size(n_seq: int, n_q: int, n_kv: int, D: int, max_keys: int) -> int:
    return int(load().blk_attn_workspace_size(n_seq, n_q, n_kv, D, max_keys))


def blk_attn_decode(q, k_cache, v_cache, block_table, lens, scale, out, ws, k_scale=None, v_scale=None,
                    stream=None):
    """q [n_seq, n_q, D]: attention of one new token of each sequence over its
    lens[s] keys in the pages block_table[s]."""
    _cache_checks(k_cache, v_cache, k_scale, v_scale)
    n_pages, n_kv, page, D = k_cache.shape
    n_seq, n_q, _ = q.shape
    _shape("q", q, n_seq, n_q, D)
    _shape("out", out, n_seq, n_q, D)
    _like("out", out, q)
    _size("lens", lens, n_seq)
    _shape("block_table", block_table, n_seq, block_table.shape[-1])
    _here(q, k_cache, v_cache, block_table, lens, out, ws, k_scale, v_scale)
    _check("blk_attn_decode", load().blk_attn_decode(
        _p(q), _dt(q), n_seq, n_q, n_kv, D, _p(k_cache), _p(v_cache), _bytes(k_scale, "e8m0"),
        _bytes(v_scale, "e8m0"), _cache_dt(k_cache, q), n_pages, page, _i32(block_table), block_table.shape[1],
        _i32(lens), float(scale), _p(out), _p(ws), ws.numel() * ws.element_size() if ws is not None else 0,
        _stream(stream)))


def blk_linear_w4(x, codes, scales, y, x_scale=None, stream=None):
    """y [T, n] = x [T, k] (bf16, float32, or 8-bit rows with x_scale) times
    the transposed 4-bit weights codes [n, k / 2], scales [n, k / 32]."""
    T, k = x.shape
    n = codes.shape[0]
    _shape("codes", codes, n, k // 2)
    _shape("scales", scales, n, k // BLOCK)
    _shape("y", y, T, n)
    _shape("x_scale", x_scale, T, k // BLOCK)
    mx = x.dtype in _BYTES["e4m3"]
    _here(x, codes, scales, y, x_scale)
    _check("blk_linear_w4", load().blk_linear_w4(
        _p(x), BLK_MX8 if mx else _dt(x), _bytes(x_scale, "e8m0"), T, k, _bytes(codes, "codes"),
        _bytes(scales, "e8m0"), n, _p(y), _dt(y), _stream(stream)))


def blk_quantize_w4(w, codes, scales, stream=None):
    """w [n, k] (bf16 or float32) -> codes [n, k / 2], scales [n, k / 32]."""
    n, k = w.shape
    _shape("codes", codes, n, k // 2)
    _shape("scales", scales, n, k // BLOCK)
    _here(w, codes, scales)
    _check("blk_quantize_w4", load().blk_quantize_w4(
        _p(w), _dt(w), n, k, _bytes(codes, "codes"), _bytes(scales, "e8m0"), _stream(stream)))


__all__ = ["MOE_BF16", "MOE_F32", "BLK_MX8", "load", *EXPORTS]
