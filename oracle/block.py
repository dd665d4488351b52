"""Plain, slow, fp64 CPU oracle of the attention half of a decoder block.

TEST INFRASTRUCTURE ONLY, like ``oracle.moe``: numpy float64 (and Python loops
over sequences and pages) on exactly widened inputs, no blocking or fusion, no
code shared with the HIP path.
"""

from __future__ import annotations

import math

import numpy as np

F64 = np.float64

#: the values of the e4m3 codes 0..127 (the last is NaN), and of the e2m1 codes 0..7
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)]
                + [np.nan])
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e8m0(byte):
    """The values of scale bytes."""
    b = np.asarray(byte).astype(np.int64)
    return np.where(b == 255, np.nan, 2.0 ** (b - 127.0))


def scale_byte(most, top):
    """The byte of the smallest 2^E, E >= -127, with most <= top * 2^E."""
    if not math.isfinite(most):
        return 255
    E = -127
    while most > top * 2.0 ** E:
        E += 1
    return E + 127


def nearest_even(v, table):
    """The index of the table's value nearest to v >= 0, ties to the even
    index (values beyond the table's end do not occur)."""
    i = int(np.searchsorted(table, v))
    if i == 0 or (i < len(table) and table[i] == v):
        return i
    if i == len(table):
        return i - 1
    lo, hi = v - table[i - 1], table[i] - v
    return i - 1 if lo < hi or (lo == hi and (i - 1) % 2 == 0) else i


def quantize_rows(v, top, table):
    """Codes (sign in the bit above the table's) and scale bytes of v [T, n]."""
    T, n = v.shape
    nb = -(-n // 32)
    codes, bytes_ = np.zeros((T, n), np.int64), np.zeros((T, nb), np.uint8)
    sign = len(table) if len(table) == 8 else 128
    for t in range(T):
        for b in range(nb):
            blk = v[t, 32 * b: 32 * b + 32]
            byte = scale_byte(float(np.max(np.abs(blk))) if np.all(np.isfinite(blk)) else math.inf, top)
            bytes_[t, b] = byte
            for j, x in enumerate(blk):
                code = len(table) - 1 if byte == 255 else nearest_even(abs(x) / e8m0(byte), table)
                codes[t, 32 * b + j] = code + (sign if np.signbit(x) and byte != 255 else 0)
    return codes, bytes_


def quantize_mx8(v):
    return quantize_rows(v, 448.0, E4M3[:127])


def quantize_w4(w):
    return quantize_rows(w, 6.0, E2M1)


def dequantize_mx8(codes, scales):
    """codes [..., n] bytes, scales [..., ceil(n / 32)] bytes -> float64."""
    c = np.asarray(codes).astype(np.int64)
    v = np.where(c >= 128, -1.0, 1.0) * E4M3[c & 127]
    return v * np.repeat(e8m0(scales), 32, axis=-1)[..., : c.shape[-1]]


def dequantize_w4(codes, scales):
    """codes [n, k / 2] bytes (even column in the low half) -> float64 [n, k]."""
    c = np.asarray(codes).astype(np.int64)
    c = np.stack([c & 15, c >> 4], -1).reshape(c.shape[0], -1)
    return np.where(c >= 8, -1.0, 1.0) * E2M1[c & 7] * np.repeat(e8m0(scales), 32, axis=-1)


def rms(v, weight, eps):
    """v / sqrt(mean(v^2) + eps) * weight over the last axis."""
    v = v.astype(F64)
    y = v / np.sqrt(np.mean(v * v, axis=-1, keepdims=True) + eps)
    return y if weight is None else y * np.asarray(weight, F64)


def rms_norm(x, residual, weight, eps):
    """(h, y): h = x + residual and its norm."""
    h = x.astype(F64) if residual is None else x.astype(F64) + residual.astype(F64)
    return h, rms(h, weight, eps)


def rotate(v, positions, inv_freq):
    """v [T, heads, D]: values i and i + r, r = len(inv_freq), turned by
    positions * inv_freq[i]."""
    r = len(inv_freq)
    a = np.asarray(positions, F64)[:, None, None] * np.asarray(inv_freq, F64)
    out = v.astype(F64).copy()
    out[..., :r] = v[..., :r] * np.cos(a) - v[..., r:2 * r] * np.sin(a)
    out[..., r:2 * r] = v[..., r:2 * r] * np.cos(a) + v[..., :r] * np.sin(a)
    return out


def heads_of(qkv, n_q, n_kv, D, q_norm, k_norm, eps, positions, inv_freq):
    """(q, k, v) [T, heads, D] of the rows qkv: head norm, then rotation."""
    rows = qkv.astype(F64).reshape(len(qkv), n_q + 2 * n_kv, D)
    q, k, v = rows[:, :n_q], rows[:, n_q:n_q + n_kv], rows[:, n_q + n_kv:]
    q = rms(q, q_norm, eps) if q_norm is not None else q
    k = rms(k, k_norm, eps) if k_norm is not None else k
    if inv_freq is not None and len(inv_freq):
        q, k = rotate(q, positions, inv_freq), rotate(k, positions, inv_freq)
    return q, k, v


def kv_extend(lens, add, n_free, table, free, page, rows_max):
    """The page tables and slot maps of a step, one sequence after the other."""
    lens, add = [int(x) for x in lens], [int(x) for x in add]
    n, width = table.shape
    n_pages = len(free)
    table, stack = table.copy(), list(int(x) for x in free)
    cap = width * page
    lens = [min(max(x, 0), cap) for x in lens]
    top = min(max(int(n_free), 0), n_pages)
    was = top
    for s in range(n):
        if add[s] < 0:
            for j in range(-(-lens[s] // page)):
                if top < n_pages:
                    stack[top] = int(table[s, j])
                    top += 1
    given = top - was
    out, offsets, accepted = list(lens), [0], [1] * n
    slots, positions = [-1] * rows_max, [0] * rows_max
    needed, taken, rows, refused, avail = 0, 0, 0, 0, top
    for s in range(n):
        if add[s] < 0:
            out[s] = 0
            offsets.append(min(rows, rows_max))
            continue
        begin, rows = rows, rows + add[s]
        offsets.append(min(rows, rows_max))
        have = -(-lens[s] // page)
        ok = lens[s] + add[s] <= cap and rows <= rows_max
        if ok:
            need = -(-(lens[s] + add[s]) // page) - have
            needed += need
            ok = need == 0 or needed <= avail
        if not ok:
            accepted[s] = 0
            refused += 1
            continue
        for j in range(need):
            top -= 1
            table[s, have + j] = stack[top]
        taken += need
        out[s] = lens[s] + add[s]
        for i in range(add[s]):
            pos = lens[s] + i
            p = int(table[s, pos // page])
            if 0 <= p < n_pages:
                slots[begin + i], positions[begin + i] = p * page + pos % page, pos
    i32 = lambda a: np.array(a, np.int32)  # noqa: E731
    return dict(len_out=i32(out), n_free_out=i32([avail - taken]), block_table=table, free_pages=i32(stack),
                row_offsets=i32(offsets), slot_map=i32(slots), positions=i32(positions), accepted=i32(accepted),
                status=i32([min(rows, rows_max), taken, refused, given]))


def keys_of(cache, table_row, length, page):
    """cache [n_pages, n_kv, page, D] float64 -> [n_kv, keys, D] of one
    sequence; keys on pages that are none are left out."""
    rows = []
    for j in range(min(max(int(length), 0), len(table_row) * page)):
        p = int(table_row[j // page])
        if 0 <= p < len(cache):
            rows.append(cache[p, :, j % page])
    return np.stack(rows, 1) if rows else np.zeros((cache.shape[1], 0, cache.shape[3]))


def attention(q, k, v, scale):
    """q [n_q, D] over k, v [n_kv, keys, D]: (out [n_q, D], the weights
    [n_q, keys]); no key, or none with a score above minus infinity: zeros."""
    n_q, D = q.shape
    group = n_q // k.shape[0]
    out, weights = np.zeros((n_q, D)), np.zeros((n_q, k.shape[1]))
    for h in range(n_q):
        s = k[h // group] @ q[h].astype(F64) * scale
        if s.size == 0 or np.max(s) == -np.inf:
            continue
        p = np.exp(s - np.max(s))
        weights[h] = p / p.sum()
        out[h] = weights[h] @ v[h // group]
    return out, weights
