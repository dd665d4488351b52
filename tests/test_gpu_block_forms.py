"""The attention half's launch forms that only certain sizes take: every tile
of the 4-bit products and their loops over several chunks, the long norms, the
cache write's runs of heads, whole-segment attention of long heads, page
tables of many sequences with few rows.  Each against the float64 oracle
through the checks of ``test_gpu_block``."""

import math

import numpy as np
import pytest
import torch

import test_gpu_block as G
from _util import U32, ensure_built, gamma
from oracle import block as O

pytestmark = pytest.mark.gpu

from paper_2609_38823_amd import block_abi as B  # noqa: E402

KINDS = [("bf16", "bf16"), ("bf16", "mx"), ("f32", "f32")]
X_KINDS = ["bf16", "mx", "f32"]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()
    B.load()
    torch.cuda.init()


# ------------------------------------------------------------- 4-bit products
@pytest.mark.parametrize("x_kind", X_KINDS)
@pytest.mark.parametrize("T", [1, 3, 4])
@pytest.mark.parametrize("k", [2304, 4128, 4192, 6176, 8224])
def test_few_rows_with_several_chunks_a_wavefront(x_kind, T, k):
    """Up to four rows, 2 to 5 chunks of 256 columns for the first wavefront,
    whole and ragged last ones."""
    G.test_linear_w4(x_kind, T, 40, k)


@pytest.mark.parametrize("x_kind", X_KINDS)
@pytest.mark.parametrize("n,k", [(8209, 96), (8209, 2336)])
def test_few_rows_of_wide_products(x_kind, n, k):
    """bf16: two groups of weight rows a workgroup; the last group is ragged."""
    G.test_linear_w4(x_kind, 2, n, k)


@pytest.mark.parametrize("x_kind", X_KINDS)
@pytest.mark.parametrize("T", [5, 16, 17, 37, 64])
@pytest.mark.parametrize("n", [4115, 8197])
def test_several_weight_groups_a_workgroup(x_kind, T, n):
    """Two and four groups of 16 weight rows for every number of row groups."""
    G.test_linear_w4(x_kind, T, n, 160)


@pytest.mark.parametrize("x_kind", X_KINDS)
@pytest.mark.parametrize("T,n,k", [(9, 33, 544), (9, 33, 2144), (17, 33, 2144), (16, 8197, 1056), (32, 4115, 1184),
                                   (48, 4115, 1184), (64, 4115, 1056), (70, 4115, 96)])
def test_chunks_and_ragged_ends(x_kind, T, n, k):
    G.test_linear_w4(x_kind, T, n, k)


# ------------------------------------------------------------------- the norm
def tight(y):
    """The bound of a float32 y that does not grow with the row: h one
    rounding; eight squares at a time, a fused product and sum each (gamma(8) of
    the mean and two roundings of h, half of it in the root), the rest of the sum
    and the root in 64 bits, eps and the factor rounded once, two products: nine
    and a half roundings and what is quadratic in them."""
    return np.abs(y) * (gamma(8) / 2 + 6 * U32) + G.TINY


@pytest.mark.parametrize("T,d", [(3, 7), (9, 512), (7, 1000), (64, 2048), (5, 4096), (33, 4100), (513, 4100), (64, 8192),
                                 (513, 8192), (2, 8200), (3, 32768)])
def test_norms_error_does_not_grow_with_the_row(T, d):
    rng = np.random.default_rng(T + d)
    x, r, w = G.rows(rng, (T, d), "f32"), G.rows(rng, (T, d), "f32", 3.0), G.rows(rng, (d,), "f32")
    h, y = torch.empty_like(x), torch.empty_like(x)
    q, qs = G.u8(T, d), G.u8(T, -(-d // 32))
    B.blk_rms_norm(x, w, 1e-6, residual=r, h_out=h, y=y, q=q, q_scale=qs)
    h64, y64 = O.rms_norm(G.host(x), G.host(r), G.host(w), 1e-6)
    assert np.all(np.abs(G.host(h) - h64) <= np.abs(h64) * U32)
    assert np.all(np.abs(G.host(y) - y64) <= tight(y64))
    pick = sorted({0, T // 2, T - 1})
    G.check_mx(q[pick], qs[pick], y64[pick], tight(y64)[pick])


@pytest.mark.parametrize("T,d", [(513, 4100), (513, 8192)])
def test_norms_of_many_long_rows_in_bf16(T, d):
    rng = np.random.default_rng(d)
    x, r, w = G.rows(rng, (T, d), "bf16"), G.rows(rng, (T, d), "bf16", 3.0), G.rows(rng, (d,), "f32")
    h, y = torch.empty_like(x), torch.empty_like(x)
    q, qs = G.u8(T, d), G.u8(T, -(-d // 32))
    B.blk_rms_norm(x, w, 1e-6, residual=r, h_out=h, y=y, q=q, q_scale=qs)
    h64, y64 = O.rms_norm(G.host(x), G.host(r), G.host(w), 1e-6)
    e = tight(y64)
    assert np.all(np.abs(G.host(h) - h64) <= np.abs(h64) * (U32 + G.EPS["bf16"] * (1 + U32)))
    assert np.all(np.abs(G.host(y) - y64) <= e + (np.abs(y64) + e) * G.EPS["bf16"])
    pick = [0, 1, 256, 511, 512]
    G.check_mx(q[pick], qs[pick], y64[pick], e[pick])


# ----------------------------------------------------- page tables and slots
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", [
    dict(n=257, page=16, width=64, longest=1000, most=1, gone=0.0, spare=300),
    dict(n=300, page=16, width=64, longest=1000, most=1, gone=0.1, spare=0),
    dict(n=600, page=8, width=40, longest=320, most=5, gone=0.1, spare=100),               # some refused
    dict(n=1024, page=16, width=8, longest=128, most=1, gone=0.0, spare=60),
    dict(n=1500, page=4, width=20, longest=80, most=1, gone=0.2, spare=50),                # two passes
    dict(n=2300, page=3, width=20, longest=60, most=1, gone=0.1, spare=2000, rows_max=700),  # rows run out
    dict(n=1100, page=5, width=12, longest=60, most=3, gone=0.1, spare=2000, rows_max=2048),
], ids=str)
def test_many_sequences_with_few_rows(case, in_place):
    """257 sequences and more with at most 2048 rows: one launch of 1024 threads."""
    args = G.extend_case(case["n"] + case["page"], **case)
    assert args[6] <= 2048
    got = G.run_extend(*args, in_place=in_place)
    ref = O.kv_extend(*args[:3], args[3].astype(np.int32), args[4].astype(np.int32), *args[5:])
    for k in ref:
        np.testing.assert_array_equal(got[k], ref[k], err_msg=k)


# -------------------------------------------------- heads and the cache write
RUNS = [(1100, 32, 4, 128, 128, 16), (2100, 32, 4, 128, 64, 64), (1300, 24, 2, 64, 64, 16), (1700, 10, 2, 256, 256, 32),
        (1500, 12, 3, 96, 96, 7), (1200, 9, 1, 192, 64, 16)]


@pytest.mark.parametrize("dt,cache", KINDS)
@pytest.mark.parametrize("T,n_q,n_kv,D,rot,page", RUNS)
def test_runs_of_heads(dt, cache, T, n_q, n_kv, D, rot, page):
    """Rows enough that a wavefront takes query, key and value heads in turn."""
    G.test_qkv_cache(dt, cache, T, n_q, n_kv, D, rot, page, True)


@pytest.mark.parametrize("dt,cache", KINDS)
@pytest.mark.parametrize("T,n_q,n_kv,D,rot,page", RUNS)
def test_runs_of_heads_give_the_bits_of_single_ones(dt, cache, T, n_q, n_kv, D, rot, page):
    """A row's values do not depend on how many heads a wavefront takes: the
    same rows a few at a time (one head group a wavefront), 8-bit rows included."""
    rng = np.random.default_rng(T)
    n_pages = T // page + 3
    x = G.rows(rng, (T, (n_q + 2 * n_kv) * D), dt)
    w = [G.rows(rng, (D,), "f32") for _ in range(2)]
    freq = torch.from_numpy((1e6 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)).cuda()
    pos, slots = G.i32(rng.integers(0, 1 << 17, T)), rng.permutation(n_pages * page)[:T]
    a = G.empty_cache(rng, n_pages, n_kv, page, D, dt, cache)
    b = [None if t is None else t.clone() for t in a]

    def call(at, arrays):
        q = torch.empty((len(at), n_q, D), dtype=G.DT[dt], device="cuda")
        pick = torch.as_tensor(at, device="cuda")
        B.blk_qkv_cache(x[pick], n_q, G.i32(slots[at]), arrays[0], arrays[1], q, positions=pos[pick], inv_freq=freq,
                        q_norm=w[0], k_norm=w[1], k_scale=arrays[2], v_scale=arrays[3])
        return q

    q = call(np.arange(T), a)
    for at in (np.arange(0, 9), np.arange(T // 2, T // 2 + 9), np.arange(T - 9, T)):
        assert G.same(call(at, b), q[at[0]:at[-1] + 1])
        pg, off = slots[at] // page, slots[at] % page
        for t, u in zip(a, b):
            if t is not None:
                np.testing.assert_array_equal(G.host(t)[pg, :, off], G.host(u)[pg, :, off])


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("dt,cache", KINDS)
@pytest.mark.parametrize("D", [192, 256])
def test_long_heads_a_segment_a_workgroup(dt, cache, D):
    """Two tiles at the most (a tile is 64 keys in float32, else 128)."""
    most = 128 if dt == "f32" else 256
    lens = [1, 0, 37, most // 2, most // 2 + 1, most]
    G.run_attn(np.random.default_rng(D), lens, 8, 2, D, 16, dt, cache, width=most // 16, poison=True)


@pytest.mark.parametrize("dt,cache", KINDS)
@pytest.mark.parametrize("n,n_q,n_kv,D,tiles", [(65, 4, 2, 64, 16), (128, 3, 1, 192, 8), (64, 8, 4, 192, 16),
                                                (33, 8, 4, 256, 8), (33, 8, 4, 256, 9)])
def test_whole_segments_of_many_tiles(dt, cache, n, n_q, n_kv, D, tiles):
    """130 to 256 segments of up to 16 tiles, both sides of the limit for long
    rows; sequences share pages."""
    rng = np.random.default_rng(n + D + tiles)
    keys = tiles * (64 if dt == "f32" else 128)
    width = keys // 16
    lens = rng.integers(0, keys + 1, n)
    lens[:4] = [keys, 0, 1, keys - 1]
    table = rng.integers(0, 40, (n, width)).astype(np.int32)
    G.run_attn(rng, lens.tolist(), n_q, n_kv, D, 16, dt, cache, width=width, table=table, n_pages=40)


def test_scale_of_an_odd_size_and_sign():
    """A scale that is no power of two, and a negative one."""
    rng = np.random.default_rng(3)
    k, v, _, _, k64, v64 = G.filled_cache(rng, 9, 2, 16, 64, "f32", "f32")
    q = G.rows(rng, (1, 4, 64), "f32")
    table = np.arange(9, dtype=np.int32)[None]
    ws = torch.empty(B.blk_attn_workspace_size(1, 4, 2, 64, 144), dtype=torch.uint8, device="cuda")
    for scale in (0.3, -0.07, 0.0):
        out = torch.empty_like(q)
        B.blk_attn_decode(q, k, v, G.i32(table), G.i32([141]), scale, out, ws)
        kk, vv = (O.keys_of(c, table[0], 141, 16) for c in (k64, v64))
        ref, w = O.attention(G.host(q)[0], kk, vv, scale)
        assert np.all(np.abs(G.host(out)[0] - ref) <= G.attn_bound(G.host(q)[0], kk, vv, w, ref, scale, "f32", 2))
