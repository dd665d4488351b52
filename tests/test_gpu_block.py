"""The attention half of a block on the GPU against the float64 oracle.

Tolerances count roundings.  u = 2^-24 is a float32 rounding, EPS[dt] a
rounding to the output's type (half a step, relative).  A float32 sum of n
terms is off by at most gamma(n) times the sum of the terms' absolute values,
in any order.
"""

import math
import os

import numpy as np
import pytest
import torch

from _util import U32, gamma
from oracle import block as O

pytestmark = pytest.mark.gpu

from paper_2609_38823_amd import abi, block_abi as B, build  # noqa: E402

EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TINY = 1e-37  # below this products and roundings may be subnormal


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(B.LIB_PATH):
        build.build()
    B.load()
    torch.cuda.init()


def host(t):
    torch.cuda.synchronize()
    if t.dtype in (torch.float8_e4m3fn, torch.float8_e8m0fnu):
        return t.view(torch.uint8).cpu().numpy()
    return t.cpu().numpy() if t.dtype in (torch.int32, torch.uint8) else t.double().cpu().numpy()


def rows(rng, shape, dt, std=1.0):
    return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32) * np.float32(std)).cuda().to(DT[dt])


def u8(*shape):
    return torch.full(shape, 0xAA, dtype=torch.uint8, device="cuda")


def i32(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def check_mx(codes, scales, ref, err):
    """8-bit rows of values within err of ref: the scale is the definition's
    for some maximum within the error, the values are within half a step."""
    codes, scales = host(codes), host(scales)
    n = ref.shape[-1]
    pad = -n % 32
    most = np.abs(np.pad(ref, [(0, 0)] * (ref.ndim - 1) + [(0, pad)])).reshape(*ref.shape[:-1], -1, 32)
    slack = np.pad(err, [(0, 0)] * (ref.ndim - 1) + [(0, pad)]).reshape(most.shape)
    for at in np.ndindex(scales.shape):
        lo = O.scale_byte(float(np.max(np.maximum(most[at] - slack[at], 0))), 448.0)
        hi = O.scale_byte(float(np.max(most[at] + slack[at])), 448.0)
        assert lo <= scales[at] <= hi, (at, lo, int(scales[at]), hi)
    step = np.repeat(O.e8m0(scales), 32, -1)[..., :n]
    got = O.dequantize_mx8(codes, scales)
    bound = np.maximum((np.abs(ref) + err) * 2.0 ** -4, step * 2.0 ** -10) + err
    assert np.all(np.abs(got - ref) <= bound)


# ------------------------------------------------------------------- the norm
def norm_bound(h, y, d):
    # h: one rounding; the mean gamma(d + 2) of a sum of squares, half of it in
    # the root; root, quotient, two products: six more
    return np.abs(y) * (gamma(d + 2) / 2 + 8 * U32) + TINY


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 1), (3, 7), (5, 32), (2, 33), (7, 250), (9, 512), (4, 513), (64, 2048), (3, 2056),
                                 (2, 4100), (3, 8192), (2, 8200), (1, 32768), (1000, 320)])
def test_rms_norm(dt, T, d):
    rng = np.random.default_rng(T * 10007 + d)
    x, r = rows(rng, (T, d), dt), rows(rng, (T, d), dt, 3.0)
    w = rows(rng, (d,), "f32")
    h, y = torch.empty_like(x), torch.empty_like(x)
    q, qs = u8(T, d).view(torch.float8_e4m3fn), u8(T, -(-d // 32)).view(torch.float8_e8m0fnu)
    B.blk_rms_norm(x, w, 1e-6, residual=r, h_out=h, y=y, q=q, q_scale=qs)
    h64, y64 = O.rms_norm(host(x), host(r), host(w), 1e-6)
    assert np.all(np.abs(host(h) - h64) <= np.abs(h64) * (U32 + EPS[dt] * (1 + U32)))
    e = norm_bound(h64, y64, d)
    assert np.all(np.abs(host(y) - y64) <= e + (np.abs(y64) + e) * EPS[dt])
    if T <= 64:
        check_mx(q, qs, y64, e)
    # without the residual and the weight, one output at a time: the same values
    h64, y64 = O.rms_norm(host(x), None, None, 1e-3)
    y2, q2, qs2 = torch.empty_like(x), torch.empty_like(q), torch.empty_like(qs)
    B.blk_rms_norm(x, None, 1e-3, y=y2)
    B.blk_rms_norm(x, None, 1e-3, q=q2, q_scale=qs2)
    e = norm_bound(h64, y64, d)
    assert np.all(np.abs(host(y2) - y64) <= e + (np.abs(y64) + e) * EPS[dt])
    if T <= 64:
        check_mx(q2, qs2, y64, e)


@pytest.mark.parametrize("T,d", [(5, 96), (300, 2048), (3, 10000)])
def test_rms_norm_in_place_and_repeated(T, d):
    rng = np.random.default_rng(d)
    x, r, w = rows(rng, (T, d), "bf16"), rows(rng, (T, d), "bf16"), rows(rng, (d,), "f32")
    h, y = torch.empty_like(x), torch.empty_like(x)
    B.blk_rms_norm(x, w, 1e-6, residual=r, h_out=h, y=y)
    h2, y2 = torch.empty_like(x), torch.empty_like(x)
    B.blk_rms_norm(x, w, 1e-6, residual=r, h_out=h2, y=y2)
    assert same(h, h2) and same(y, y2)
    xa, ra = x.clone(), r.clone()
    B.blk_rms_norm(xa, w, 1e-6, residual=ra, h_out=ra, y=xa)
    assert same(ra, h) and same(xa, y)
    xa = x.clone()
    B.blk_rms_norm(xa, w, 1e-6, residual=xa, h_out=xa, y=y2)  # x + x
    assert np.array_equal(host(xa), 2 * host(x))


def test_rms_norm_of_zeros_infinities_and_nans():
    x = torch.zeros((4, 64), device="cuda")
    x[1, 3], x[2, 40], x[3] = math.inf, math.nan, 1e-30
    q, qs = u8(4, 64), u8(4, 2)
    y = torch.empty_like(x)
    B.blk_rms_norm(x, None, 0.0, y=y, q=q, q_scale=qs)
    with np.errstate(all="ignore"):
        _, ref = O.rms_norm(host(x), None, None, 0.0)
    got = host(y)
    # all zeros with eps 0: 0 / 0; an infinity makes itself NaN and the others 0
    assert np.isnan(got[0]).all() and np.isnan(got[1, 3]) and not got[1, np.arange(64) != 3].any()
    assert np.isnan(got[2]).all() and np.isnan(ref[2]).all()
    s = host(qs)
    assert s[0].tolist() == [255, 255] and s[1].tolist() == [255, 0] and s[2].tolist() == [255, 255]
    assert np.isnan(O.dequantize_mx8(host(q)[2], s[2])).all()
    B.blk_rms_norm(x[:1], None, 1e-6, y=y[:1], q=q[:1], q_scale=qs[:1])
    assert not host(y)[0].any() and host(qs)[0].tolist() == [0, 0] and not host(q)[0].any()


# ----------------------------------------------------- page tables and slots
def run_extend(lens, add, n_free, table, free, page, rows_max, in_place=False):
    n = len(lens)
    t, f = i32(table), i32(free)
    li, nf = i32(lens), i32([n_free])
    lo, nfo = (li, nf) if in_place else (i32([-7] * n), i32([-7]))
    off, slots, pos = i32([-7] * (n + 1)), i32([-7] * rows_max), i32([-7] * rows_max)
    acc, st = i32([-7] * n), i32([-7] * 4)
    B.blk_kv_extend(li, i32(add), nf, t, f, page, lo, nfo, off, slots, pos, acc, st)
    return dict(len_out=host(lo), n_free_out=host(nfo), block_table=host(t), free_pages=host(f),
                row_offsets=host(off), slot_map=host(slots), positions=host(pos), accepted=host(acc), status=host(st))


def extend_case(seed, n, page, width, longest, most, gone, spare, rows_max=None):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, min(longest, width * page) + 1, n)
    add = np.where(rng.random(n) < gone, -1, rng.integers(0, most + 1, n))
    have = -(-lens // page)
    n_pages = int(have.sum()) + spare
    perm = rng.permutation(max(n_pages, 1))
    table, at = np.full((n, width), -1), 0
    for s in range(n):
        table[s, :have[s]] = perm[at:at + have[s]]
        at += have[s]
    free = np.concatenate([perm[at:], np.full(at, -3)])[:max(n_pages, 1)]
    return lens, add, max(n_pages, 1) - at if n_pages else 0, table, free, page, \
        int(add.clip(0).sum()) + 5 if rows_max is None else rows_max


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", [
    dict(n=1, page=16, width=4, longest=40, most=1, gone=0.0, spare=4),
    dict(n=1, page=1, width=300, longest=100, most=200, gone=0.0, spare=200),
    dict(n=64, page=16, width=64, longest=1000, most=1, gone=0.0, spare=64),
    dict(n=64, page=16, width=64, longest=1000, most=1, gone=0.2, spare=0),       # only the finished ones' pages
    dict(n=64, page=8, width=40, longest=320, most=60, gone=0.1, spare=100),      # some refused for room or pages
    dict(n=200, page=3, width=30, longest=80, most=40, gone=0.3, spare=300, rows_max=1000),  # rows run out
    dict(n=1025, page=16, width=8, longest=100, most=20, gone=0.1, spare=500),    # more than one pass
    dict(n=3000, page=4, width=6, longest=24, most=6, gone=0.4, spare=10),
    dict(n=50, page=64, width=50, longest=1000, most=2000, gone=0.1, spare=3000),  # many rows
    dict(n=2100, page=16, width=9, longest=60, most=80, gone=0.1, spare=4000),
    dict(n=7, page=5, width=9, longest=45, most=0, gone=0.0, spare=3),            # nothing to append
    dict(n=5, page=7, width=3, longest=21, most=3, gone=1.0, spare=2),            # all finished
], ids=str)
def test_kv_extend(case, in_place):
    args = extend_case(case["n"] * 31 + case["page"], **case)
    got, ref = run_extend(*args, in_place=in_place), O.kv_extend(*[args[i] for i in (0, 1, 2)], args[3].astype(np.int32),
                                                                 args[4].astype(np.int32), *args[5:])
    for k in ref:
        np.testing.assert_array_equal(got[k], ref[k], err_msg=k)


def test_kv_extend_of_no_sequence_and_no_row():
    got = run_extend([], [], 3, np.zeros((0, 2), np.int32), np.arange(4), 4, 9)
    assert (got["slot_map"] == -1).all() and got["row_offsets"].tolist() == [0] and got["n_free_out"].tolist() == [3]
    got = run_extend([4, 3], [0, 0], 3, np.zeros((2, 2), np.int32), np.arange(4), 4, 0)
    assert got["accepted"].tolist() == [1, 1] and got["row_offsets"].tolist() == [0, 0, 0]
    got = run_extend([4, 3], [1, 1], 3, np.zeros((2, 2), np.int32), np.arange(4), 4, 0)
    assert got["accepted"].tolist() == [0, 0] and got["len_out"].tolist() == [4, 3]


def test_kv_extend_clamps_what_is_out_of_range():
    """Lengths, free counts and page entries that are none: no access leaves
    an array, and the oracle's result."""
    table = np.array([[5, 900], [-4, 1], [2, 3]], np.int32)
    free = np.array([0, 77, 4, 6, 7, 7, 7, 7], np.int32)
    for n_free in (-5, 2, 100):
        a = ([3, 1000, -9], [3, -2, 2], n_free, table, free, 4, 12)
        got, ref = run_extend(*a), O.kv_extend(*a)
        for k in ref:
            np.testing.assert_array_equal(got[k], ref[k], err_msg=k)
    big = (1 << 31) - 1
    a = ([3, 1], [big, big], 4, table[:2], free, 4, 12)
    got = run_extend(*a)
    assert got["accepted"].tolist() == [0, 0] and got["row_offsets"].tolist() == [0, 12, 12]


# -------------------------------------------------- heads and the cache write
def empty_cache(rng, n_pages, n_kv, page, D, dt, cache):
    if cache == "mx":
        bytes_ = lambda *s: torch.from_numpy(rng.integers(0, 120, s).astype(np.uint8)).cuda()  # noqa: E731
        return [bytes_(n_pages, n_kv, page, D), bytes_(n_pages, n_kv, page, D),
                bytes_(n_pages, n_kv, page, D // 32), bytes_(n_pages, n_kv, page, D // 32)]
    return [rows(rng, (n_pages, n_kv, page, D), dt), rows(rng, (n_pages, n_kv, page, D), dt), None, None]


@pytest.mark.parametrize("dt,cache", [("bf16", "bf16"), ("bf16", "mx"), ("f32", "f32")])
@pytest.mark.parametrize("T,n_q,n_kv,D,rot,page,norm", [
    (1, 1, 1, 32, 0, 1, False), (3, 8, 2, 64, 64, 16, True), (7, 32, 4, 128, 128, 16, True),
    (5, 5, 1, 96, 96, 3, True), (2, 6, 6, 192, 64, 8, False), (4, 4, 2, 256, 256, 10, True),
    (6, 3, 3, 160, 32, 7, True), (33, 16, 1, 224, 224, 5, False), (4100, 2, 1, 32, 16, 64, True)])
def test_qkv_cache(dt, cache, T, n_q, n_kv, D, rot, page, norm):
    rng = np.random.default_rng(T * 100 + D)
    n_pages = T // page + 3
    x = rows(rng, (T, (n_q + 2 * n_kv) * D), dt)
    w = [rows(rng, (D,), "f32") for _ in range(2)] if norm else [None, None]
    pos = rng.integers(0, 1 << 20, T)
    pos[0] = (1 << 31) - 1
    freq = (1e6 ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)
    slots = rng.permutation(n_pages * page)[:T]
    if T > 2:
        slots[1], slots[2] = -1, n_pages * page  # no slot: not written
    kc, vc, ks, vs = empty_cache(rng, n_pages, n_kv, page, D, dt, cache)
    before = [None if t is None else t.clone() for t in (kc, vc, ks, vs)]
    q = torch.empty((T, n_q, D), dtype=DT[dt], device="cuda")
    B.blk_qkv_cache(x, n_q, i32(slots), kc, vc, q, positions=i32(pos),
                    inv_freq=torch.from_numpy(freq).cuda() if rot else None, q_norm=w[0], k_norm=w[1], eps=1e-6,
                    k_scale=ks, v_scale=vs)
    x64, w64 = host(x), [None if t is None else host(t) for t in w]
    q64, k64, v64 = O.heads_of(x64, n_q, n_kv, D, w64[0], w64[1], 1e-6, pos, freq if rot else None)
    # the norm as in blk_rms_norm; a rotated value is a cos + b sin with |a| + |b|
    # times: two products and a sum (3 u), the angle's fraction of a turn in
    # float32 (pi u) and the sine and cosine themselves (2 u)
    plain = O.heads_of(x64, n_q, n_kv, D, w64[0], w64[1], 1e-6, pos, None)
    errs = []
    for v, p in ((q64, plain[0]), (k64, plain[1])):
        e = np.abs(p) * (gamma(D + 2) / 2 + 8 * U32) if norm else np.zeros_like(p)
        both, ee = np.abs(p).copy(), e.copy()
        r = rot // 2
        both[..., :r] += np.abs(p[..., r:rot])
        both[..., r:rot] += np.abs(p[..., :r])
        ee[..., :r] += e[..., r:rot]
        ee[..., r:rot] += e[..., :r]
        errs.append(ee + (both * (math.pi + 6) * U32 if rot else 0) + TINY)
    assert np.all(np.abs(host(q) - q64) <= errs[0] + (np.abs(q64) + errs[0]) * EPS[dt])
    ok = (slots >= 0) & (slots < n_pages * page)
    at, off = slots[ok] // page, slots[ok] % page
    untouched = np.ones((n_pages, page), bool)
    untouched[at, off] = False
    for c, s, b, bs, ref, err in ((kc, ks, before[0], before[2], k64[ok], errs[1][ok]),
                                  (vc, vs, before[1], before[3], v64[ok], np.zeros_like(v64[ok]))):
        got = host(c)[at, :, off]
        if cache == "mx":
            if T <= 64:
                check_mx(torch.from_numpy(got).cuda(), torch.from_numpy(host(s)[at, :, off]).cuda(), ref, err)
            np.testing.assert_array_equal(host(s).swapaxes(1, 2)[untouched], host(bs).swapaxes(1, 2)[untouched])
        else:
            assert np.all(np.abs(got - ref) <= err + (np.abs(ref) + err) * EPS[dt])
        np.testing.assert_array_equal(host(c).swapaxes(1, 2)[untouched], host(b).swapaxes(1, 2)[untouched])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_qkv_cache_leaves_columns_behind_the_rotation_alone(dt):
    """Values from rot on and the value heads pass as they are, infinities too;
    a NaN position angle does not exist, a NaN value stays in its own pair."""
    D, rot = 64, 32
    x = torch.zeros((2, 3 * D), device="cuda").to(DT[dt])
    x[0, 40], x[0, D + 63], x[0, 2 * D + 5] = math.inf, -math.inf, math.nan
    x[1, 3], x[1, D + 20] = math.nan, math.inf
    kc, vc, _, _ = empty_cache(np.random.default_rng(0), 1, 1, 4, D, dt, dt)
    q = torch.empty((2, 1, D), dtype=DT[dt], device="cuda")
    B.blk_qkv_cache(x, 1, i32([2, 0]), kc, vc, q, positions=i32([7, 0]), inv_freq=torch.ones(rot // 2, device="cuda"))
    q, k, v = host(q), host(kc)[0, 0, [2, 0]], host(vc)[0, 0, [2, 0]]
    assert q[0, 0, 40] == math.inf and not np.delete(q[0, 0], 40).any()
    assert k[0, 63] == -math.inf and not np.delete(k[0], 63).any() and np.isnan(v[0, 5]) and not np.delete(v[0], 5).any()
    assert np.isnan(q[1, 0, [3, 19]]).all() and not np.delete(q[1, 0], [3, 19]).any()
    assert not np.isfinite(k[1, [4, 20]]).any() and not np.delete(k[1], [4, 20]).any() and not v[1].any()


# ------------------------------------------------------------------ attention
def filled_cache(rng, n_pages, n_kv, page, D, dt, cache, std=1.0):
    """The cache's arrays and their values in float64."""
    if cache != "mx":
        k, v = rows(rng, (n_pages, n_kv, page, D), dt, std), rows(rng, (n_pages, n_kv, page, D), dt)
        return k, v, None, None, host(k), host(v)
    out = []
    for _ in range(2):
        codes = rng.integers(0, 256, (n_pages, n_kv, page, D)).astype(np.uint8)
        codes[(codes & 127) == 127] = 0
        scales = rng.integers(115, 123, (n_pages, n_kv, page, D // 32)).astype(np.uint8)
        out.append((codes, scales))
    (kc, ks), (vc, vs) = out
    put = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    return put(kc), put(vc), put(ks), put(vs), O.dequantize_mx8(kc, ks), O.dequantize_mx8(vc, vs)


def attn_bound(q, k, v, w, out, scale, dt, group):
    """A score is a float32 sum of D exact (bf16) or rounded products, times
    the scale (rounded) : (gamma(D + 4)) sum |q k| |scale|; its exponential is
    off by that and a few u of the exponent's own size; with bf16 keys each
    term is rounded to bf16, in the sum and in the product alike; the sums over
    the keys, rescaled at most once a step, and the join: gamma of the keys."""
    n_q, D = q.shape
    keys = k.shape[1]
    bound = np.zeros_like(out)
    for h in range(n_q):
        kk, vv = k[h // group], v[h // group]
        if not keys:
            continue
        s = np.abs(kk) @ np.abs(q[h]) * abs(scale)
        ds = (gamma(D + 4) * np.max(s) + 4 * U32 * np.max(s)) + 4 * U32
        term = math.expm1(ds) + (EPS["bf16"] if dt == "bf16" else 0.0)
        sums = 2 * gamma(keys + 2 * (keys // 16) + 64)
        bound[h] = (w[h] @ np.abs(vv)) * ((1 + term) / (1 - term) - 1 + sums)
    return bound + (np.abs(out) + bound) * EPS[dt] + TINY


def run_attn(rng, lens, n_q, n_kv, D, page, dt, cache, width=None, table=None, n_pages=None, std=1.0, poison=False):
    n = len(lens)
    width = width or max(1, -(-max(max(lens), 1) // page))
    n_pages = n_pages or n * width + 1
    kc, vc, ks, vs, k64, v64 = filled_cache(rng, n_pages, n_kv, page, D, dt, cache, std)
    if table is None:
        table = rng.permutation(n_pages)[:n * width].reshape(n, width)
    if poison:  # what no sequence reaches holds NaN, infinities and the types' largest values
        used = np.zeros((n_pages, page), bool)
        for s in range(n):
            for j in range(lens[s]):
                used[table[s, j // page], j % page] = True
        idle = torch.from_numpy(~used).cuda()
        bad = [math.nan, math.inf, -math.inf, 3e38]
        for t, fill in ((kc, bad), (vc, bad)) if cache != "mx" else ((kc, [127, 255]), (vc, [127, 255]), (ks, [255]),
                                                                       (vs, [255])):
            values = torch.tensor(fill, device="cuda", dtype=t.dtype)
            pick = torch.randint(0, len(fill), t.shape, device="cuda")
            t.copy_(torch.where(idle[:, None, :, None], values[pick], t))
    q = rows(rng, (n, n_q, D), dt, std)
    out = torch.full((n, n_q, D), 7.0, dtype=DT[dt], device="cuda")
    ws = torch.full((B.blk_attn_workspace_size(n, n_q, n_kv, D, width * page),), 0x7F, dtype=torch.uint8, device="cuda")
    scale = D ** -0.5
    call = lambda o: B.blk_attn_decode(q, kc, vc, i32(table), i32(lens), scale, o, ws, k_scale=ks, v_scale=vs)  # noqa: E731
    call(out)
    got, q64 = host(out), host(q)
    for s in range(n):
        k, v = (O.keys_of(c, table[s], lens[s], page) for c in (k64, v64))
        ref, w = O.attention(q64[s], k, v, scale)
        assert np.all(np.abs(got[s] - ref) <= attn_bound(q64[s], k, v, w, ref, scale, dt, n_q // n_kv)), s
    again = torch.empty_like(out)
    call(again)
    torch.cuda.synchronize()
    assert same(out, again)


KINDS = [("bf16", "bf16"), ("bf16", "mx"), ("f32", "f32")]


@pytest.mark.parametrize("dt,cache", KINDS)
@pytest.mark.parametrize("D", [32, 64, 96, 128, 192, 256])
def test_attn_head_lengths(dt, cache, D):
    run_attn(np.random.default_rng(D), [1, 0, 37, 128, 129, 300], 8, 2, D, 16, dt, cache)


@pytest.mark.parametrize("dt,cache", KINDS)
@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (3, 1), (8, 8), (16, 1), (17, 1), (40, 2), (128, 2)])
def test_attn_groups(dt, cache, n_q, n_kv):
    run_attn(np.random.default_rng(n_q), [65, 200, 3], n_q, n_kv, 64, 8, dt, cache)


@pytest.mark.parametrize("dt,cache", KINDS)
@pytest.mark.parametrize("page", [1, 2, 3, 5, 16, 33, 64, 100, 1000])
def test_attn_pages(dt, cache, page):
    run_attn(np.random.default_rng(page), [1, page, page + 1, 257, 64, 0], 4, 1, 64, page, dt, cache)


@pytest.mark.parametrize("dt,cache", KINDS)
def test_attn_split_over_the_length(dt, cache):
    # one long sequence among short ones: its keys are cut over many workgroups
    run_attn(np.random.default_rng(5), [20001, 5, 0, 700], 8, 2, 128, 16, dt, cache)
    run_attn(np.random.default_rng(6), [9000], 2, 1, 64, 64, dt, cache)


@pytest.mark.parametrize("dt,cache", KINDS)
@pytest.mark.parametrize("D,n_q,n_kv,page", [(32, 4, 4, 7), (64, 17, 1, 16), (96, 12, 3, 16), (128, 40, 2, 64), (192, 6, 1, 33),
                                             (256, 8, 2, 16)])
def test_attn_runs(dt, cache, D, n_q, n_kv, page):
    """Tables wide enough for the runs that cut the tiles of all sequences,
    whatever their lengths are: none, one key, parts of tiles, many tiles."""
    run_attn(np.random.default_rng(D + n_q), [0, 1, 1500, 129, 0, 640, 33, 2], n_q, n_kv, D, page, dt, cache,
             width=2000 // page + 1, poison=D in (64, 128))


@pytest.mark.parametrize("dt,cache", KINDS)
def test_attn_runs_of_many_sequences(dt, cache):
    """More segments than runs, and lengths that leave most runs several."""
    rng = np.random.default_rng(17)
    lens = rng.integers(0, 40, 600).tolist()
    lens[77], lens[500] = 3000, 2100
    run_attn(rng, lens, 4, 2, 64, 64, dt, cache, width=50)


@pytest.mark.parametrize("dt,cache", KINDS)
def test_attn_many_sequences(dt, cache):
    rng = np.random.default_rng(7)
    run_attn(rng, rng.integers(0, 200, 700).tolist(), 4, 2, 32, 16, dt, cache)


@pytest.mark.parametrize("dt,cache", KINDS)
def test_attn_uses_nothing_behind_the_last_key(dt, cache):
    run_attn(np.random.default_rng(8), [1, 0, 31, 33, 127, 140, 261], 8, 2, 64, 16, dt, cache, width=20, poison=True)


@pytest.mark.parametrize("dt,cache", KINDS)
def test_attn_large_scores(dt, cache):
    """Scores of some hundreds: all but one term vanish, and the running
    maximum rises many times."""
    run_attn(np.random.default_rng(9), [400, 63], 4, 4, 64, 16, dt, cache, std=8.0)


def test_attn_shared_and_bad_pages():
    """Sequences that share pages; entries that are no page are left out;
    lengths beyond the table and below zero are clamped."""
    rng = np.random.default_rng(10)
    table = np.array([[3, 1, 2], [3, 1, 0], [-1, 4, 1 << 30], [7, -2, 9], [0, 0, 0]], np.int32)
    run_attn(rng, [40, 48, 48, 20, 10], 4, 2, 64, 16, "bf16", "bf16", width=3, table=table, n_pages=5)
    k, v, _, _, k64, v64 = filled_cache(rng, 5, 2, 16, 64, "f32", "f32")
    q = rows(rng, (2, 4, 64), "f32")
    out = torch.empty_like(q)
    ws = torch.empty(B.blk_attn_workspace_size(2, 4, 2, 64, 48), dtype=torch.uint8, device="cuda")
    B.blk_attn_decode(q, k, v, i32(table[:2]), i32([1000, -3]), 0.125, out, ws)
    kk, vv = (O.keys_of(c, table[0], 48, 16) for c in (k64, v64))
    ref, w = O.attention(host(q)[0], kk, vv, 0.125)
    got = host(out)
    assert np.all(np.abs(got[0] - ref) <= attn_bound(host(q)[0], kk, vv, w, ref, 0.125, "f32", 2)) and not got[1].any()


def test_attn_infinite_scores():
    """-inf scores have no weight; a row of them alone gives zeros; a NaN key
    or query reaches the rows that see it and no others."""
    rng = np.random.default_rng(11)
    k, v, _, _, k64, v64 = filled_cache(rng, 6, 1, 16, 32, "f32", "f32")
    q = torch.zeros((4, 1, 32), device="cuda")
    q[:, 0, 0] = 1.0
    k[0, 0, :, 0] = -math.inf          # sequence 0: no key left
    k[1, 0, ::2, 0] = -math.inf        # sequence 1: every other one
    k[2, 0, 3, 0] = math.nan
    q[3, 0, 5] = math.nan
    out = torch.empty_like(q)
    ws = torch.empty(B.blk_attn_workspace_size(4, 1, 1, 32, 16), dtype=torch.uint8, device="cuda")
    B.blk_attn_decode(q, k, v, i32([[0], [1], [2], [3]]), i32([16, 16, 16, 16]), 1.0, out, ws)
    got = host(out)
    assert not got[0].any() and np.isfinite(got[1]).all() and np.isnan(got[2]).all() and np.isnan(got[3]).all()
    kk, vv = host(k)[1, :, 1::2], v64[1, :, 1::2]
    ref, w = O.attention(host(q)[1], kk, vv, 1.0)
    assert np.all(np.abs(got[1] - ref) <= attn_bound(host(q)[1], kk, vv, w, ref, 1.0, "f32", 1))


# ------------------------------------------------------------- 4-bit products
@pytest.mark.parametrize("x_kind", ["bf16", "mx", "f32"])
@pytest.mark.parametrize("T,n,k", [(1, 1, 32), (1, 16, 128), (2, 17, 96), (5, 100, 160), (16, 64, 512), (17, 33, 2048),
                                   (33, 130, 544), (64, 48, 256), (65, 40, 384), (130, 31, 1056), (1, 5120, 2048),
                                   (9, 250, 7168)])
def test_linear_w4(x_kind, T, n, k):
    rng = np.random.default_rng(T * 7 + n + k)
    codes = rng.integers(0, 256, (n, k // 2)).astype(np.uint8)
    scales = rng.integers(110, 125, (n, k // 32)).astype(np.uint8)
    w64 = O.dequantize_w4(codes, scales)
    xs = None
    if x_kind == "mx":
        xc, sc = rng.integers(0, 256, (T, k)).astype(np.uint8), rng.integers(115, 130, (T, k // 32)).astype(np.uint8)
        xc[(xc & 127) == 127] = 1
        x64, x, xs = O.dequantize_mx8(xc, sc), torch.from_numpy(xc).cuda(), torch.from_numpy(sc).cuda()
    else:
        x = rows(rng, (T, k), x_kind)
        x64 = host(x)
    ref, size = x64 @ w64.T, np.abs(x64) @ np.abs(w64.T)
    lost = np.zeros_like(ref)
    if x_kind == "mx":
        # the scaled matrix instruction aligns the products of eight neighbouring
        # columns to the largest of their exponents and keeps 13 bits below it: a
        # product a 2^i * b 2^j, 1 <= a, b < 2, has the exponent i + j and is at
        # least 2^(i + j), so each of the other seven loses less than 2^-13 of
        # the largest product
        for g in range(k // 8):
            part = np.s_[:, 8 * g: 8 * g + 8]
            lost += 7 * 2.0 ** -13 * np.max(np.abs(x64[part])[:, None] * np.abs(w64[part])[None], -1)
    for out in ("bf16", "f32"):
        y = torch.full((T, n), 7.0, dtype=DT[out], device="cuda")
        B.blk_linear_w4(x, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), y, x_scale=xs)
        e = size * gamma(k + 4) + lost  # products (exact but for float32 x) and a sum of k
        assert np.all(np.abs(host(y) - ref) <= e + (np.abs(ref) + e) * EPS[out] + TINY), out


def test_linear_w4_scales_at_the_ends():
    """Scale bytes 0, 1, 254 and 255 (NaN), of weights and of rows."""
    k, n = 128, 16
    codes = torch.full((n, k // 2), 0x22, dtype=torch.uint8, device="cuda")  # ones
    scales = torch.full((n, 4), 127, dtype=torch.uint8, device="cuda")
    scales[1] = 255
    scales[2] = 254
    scales[3] = 1
    x = torch.ones((1, k), device="cuda")
    xc = x.to(torch.float8_e4m3fn)
    xs = torch.full((1, 4), 127, dtype=torch.uint8, device="cuda")
    for args in ((x, None), (x.bfloat16(), None), (xc, xs)):
        y = torch.empty((1, n), device="cuda")
        B.blk_linear_w4(args[0], codes, scales, y, x_scale=args[1])
        got = host(y)[0]
        assert got[0] == 128 and np.isnan(got[1]) and got[2] == math.inf and got[3] == 2.0 ** -119, args[0].dtype
        assert (got[4:] == 128).all()
    xs[0, 2] = 255
    B.blk_linear_w4(xc, codes, scales, y, x_scale=xs)
    assert np.isnan(host(y)).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n,k", [(1, 32), (7, 96), (50, 1024)])
def test_quantize_w4(dt, n, k):
    rng = np.random.default_rng(n + k)
    w = rows(rng, (n, k), dt, 0.02)
    w[0, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -6.0], device="cuda").to(DT[dt])
    if n > 5:
        w[1, :32], w[2, 5], w[3, 70], w[4] = 0.0, math.inf, math.nan, 0.0
        w[4, 40] = 2.0 ** -126
    codes, scales = u8(n, k // 2), u8(n, k // 32)
    B.blk_quantize_w4(w, codes, scales)
    c, s = O.quantize_w4(host(w))
    got = host(codes)
    got = np.stack([got & 15, got >> 4], -1).reshape(n, k)
    np.testing.assert_array_equal(host(scales), s)
    fine = np.repeat(s, 32, 1) != 255  # the codes of a block that is not finite say nothing
    np.testing.assert_array_equal(got[fine], c[fine])


# ------------------------------------------------------- streams and refusals
def test_calls_on_another_stream_and_in_a_graph():
    """A step on a side stream, captured with its lengths advancing in place,
    replayed several times between eager work, against eager calls."""
    rng = np.random.default_rng(12)
    n, n_q, n_kv, D, page, width = 5, 8, 2, 64, 4, 6
    x = rows(rng, (n, (n_q + 2 * n_kv) * D), "bf16")
    kc, vc = (torch.zeros((n * width, n_kv, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    freq = torch.from_numpy((1e4 ** (-np.arange(0, D, 2) / D)).astype(np.float32)).cuda()

    def state():
        return dict(len=i32([0] * n), nf=i32([n * width]), table=i32(np.full((n, width), -1)), free=i32(np.arange(n * width)),
                    off=i32([0] * (n + 1)), slots=i32([0] * n), pos=i32([0] * n), acc=i32([0] * n), st=i32([0] * 4),
                    add=i32([1, 1, 0, 1, 1]), k=kc.clone(), v=vc.clone(), q=torch.empty((n, n_q, D), dtype=torch.bfloat16, device="cuda"),
                    out=torch.empty((n, n_q, D), dtype=torch.bfloat16, device="cuda"),
                    ws=torch.empty(B.blk_attn_workspace_size(n, n_q, n_kv, D, width * page), dtype=torch.uint8, device="cuda"))

    def step(s, stream=None):
        B.blk_kv_extend(s["len"], s["add"], s["nf"], s["table"], s["free"], page, s["len"], s["nf"], s["off"], s["slots"],
                        s["pos"], s["acc"], s["st"], stream=stream)
        B.blk_qkv_cache(x, n_q, s["slots"], s["k"], s["v"], s["q"], positions=s["pos"], inv_freq=freq, stream=stream)
        B.blk_attn_decode(s["q"], s["k"], s["v"], s["table"], s["len"], 0.125, s["out"], s["ws"], stream=stream)

    a, b, c = state(), state(), state()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step(b)
    side = torch.cuda.Stream()
    for i in range(9):
        step(a)
        g.replay()
        torch.cuda.synchronize()
        step(c, stream=side)
        side.synchronize()
        for k in ("len", "nf", "table", "slots", "pos", "out", "k", "v", "q", "acc", "st"):
            assert torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]), (i, k)
    assert host(a["len"]).tolist() == [9, 9, 0, 9, 9]


def test_binding_refuses_mismatched_arrays():
    x = torch.zeros((4, 64), device="cuda")
    with pytest.raises(ValueError):
        B.blk_rms_norm(x, None, 1e-6, y=torch.zeros((4, 32), device="cuda"))
    with pytest.raises(TypeError):
        B.blk_rms_norm(x, None, 1e-6, y=x.bfloat16())
    with pytest.raises(ValueError):
        B.blk_rms_norm(x.t(), None, 1e-6, y=torch.zeros((64, 4), device="cuda"))
    with pytest.raises(ValueError):
        B.blk_linear_w4(x, u8(8, 32), u8(8, 1), torch.zeros((4, 8), device="cuda"))
    with pytest.raises(TypeError):
        B.blk_linear_w4(x, x[:, :32].contiguous(), u8(4, 2), torch.zeros((4, 4), device="cuda"))
    with pytest.raises(abi.MoeError):
        B.blk_rms_norm(x, None, -1.0, y=torch.zeros_like(x))
