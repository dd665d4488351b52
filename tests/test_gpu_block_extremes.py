"""The attention half at the ends of the number range and of its precision:
softmax weights that are not rounded to the rows' type, norms of values whose
squares leave float32, rows without weight over values that are not finite."""

import math

import numpy as np
import pytest
import torch

import test_gpu_block as G
from _util import U32, ensure_built, gamma
from oracle import block as O

pytestmark = pytest.mark.gpu

from paper_2609_38823_amd import block_abi as B  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()
    B.load()
    torch.cuda.init()


# ------------------------------------------------------------------ attention
def weights_bound(q, k, v, w, out, scale, group):
    """``attn_bound`` with softmax weights in two bf16 parts: what a weight p
    leaves after its first, |p - a| <= 2^-8 p, is rounded to bf16 again, 2^-16 of
    p at most; the sum is of the unrounded weights."""
    n_q, D = q.shape
    keys = k.shape[1]
    bound = np.zeros_like(out)
    for h in range(n_q):
        kk, vv = k[h // group], v[h // group]
        s = np.max(np.abs(kk) @ np.abs(q[h]) * abs(scale))
        term = math.expm1((gamma(D + 4) + 4 * U32) * s + 4 * U32) + 2.0 ** -16
        sums = 2 * gamma(keys + 2 * (keys // 16) + 64)
        bound[h] = (w[h] @ np.abs(vv)) * ((1 + term) / (1 - term) - 1 + sums)
    return bound + (np.abs(out) + bound) * G.EPS["bf16"] + G.TINY


@pytest.mark.parametrize("cache", ["bf16", "mx"])
@pytest.mark.parametrize("keys,width,n_q,n_kv,D", [(300, 20, 8, 2, 64), (300, 20, 5, 1, 32), (500, 32, 16, 2, 128),
                                                   (250, 16, 4, 1, 256), (400, 200, 6, 2, 96), (2000, 128, 8, 1, 128),
                                                   (700, 64, 4, 1, 192)])
def test_softmax_weights_keep_more_than_the_rows_type(cache, keys, width, n_q, n_kv, D):
    """Whole segments and runs: results that are small next to the values they
    are made of show the weights' precision."""
    rng = np.random.default_rng(keys + D)
    k, v, ks, vs, k64, v64 = G.filled_cache(rng, width, n_kv, 16, D, "bf16", cache, 0.5)
    table = rng.permutation(width)[None].astype(np.int32)
    q = G.rows(rng, (1, n_q, D), "bf16", 0.5)
    out = torch.empty_like(q)
    ws = torch.empty(B.blk_attn_workspace_size(1, n_q, n_kv, D, width * 16), dtype=torch.uint8, device="cuda")
    scale = D ** -0.5
    B.blk_attn_decode(q, k, v, G.i32(table), G.i32([keys]), scale, out, ws, k_scale=ks, v_scale=vs)
    kk, vv = (O.keys_of(c, table[0], keys, 16) for c in (k64, v64))
    ref, w = O.attention(G.host(q)[0], kk, vv, scale)
    assert np.all(np.abs(G.host(out)[0] - ref) <= weights_bound(G.host(q)[0], kk, vv, w, ref, scale, n_q // n_kv))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("width", [4, 400])
def test_a_row_without_weight_gives_zeros_over_any_values(dt, width):
    """All scores minus infinity: zeros, also where the values are infinities
    or NaN, in one workgroup's segment and in one that several share."""
    n_kv, D, page = 1, 64, 16
    k, v, _, _, _, _ = G.filled_cache(np.random.default_rng(1), width, n_kv, page, D, dt, dt)
    k[..., 0] = -math.inf
    v[..., ::3], v[..., 1::3] = math.inf, math.nan
    q = torch.zeros((1, 2, D), device="cuda").to(G.DT[dt])
    q[..., 0] = 1.0
    out = torch.full_like(q, 7.0)
    ws = torch.empty(B.blk_attn_workspace_size(1, 2, n_kv, D, width * page), dtype=torch.uint8, device="cuda")
    B.blk_attn_decode(q, k, v, torch.arange(width, dtype=torch.int32, device="cuda")[None], G.i32([width * page]), 1.0,
                      out, ws)
    assert not G.host(out).any()


# ------------------------------------------------------------------ the norms
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [5, 64, 320, 1000, 4096, 6000, 9000])
def test_norm_of_rows_whose_squares_leave_float32(dt, d):
    """Values of 1e-36 to 1e37 with eps 0 or none that counts: the norm is of
    size one all the same."""
    rng = np.random.default_rng(d)
    sizes = [1e37, 1e30, 3e19, 1e18, 1.0, 1e-18, 1e-21, 1e-25, 1e-36]
    x = G.rows(rng, (len(sizes), d), "f32")
    x = (x.double() * torch.tensor(sizes, device="cuda").double()[:, None]).to(G.DT[dt])
    w = G.rows(rng, (d,), "f32")
    h, y = torch.empty_like(x), torch.empty_like(x)
    q, qs = G.u8(len(sizes), d), G.u8(len(sizes), -(-d // 32))
    B.blk_rms_norm(x, w, 0.0, h_out=h, y=y, q=q, q_scale=qs)
    assert G.same(h, x)
    _, y64 = O.rms_norm(G.host(x), None, G.host(w), 0.0)
    # eight squares at a time in float32, the rest in 64 bits; the factor, the
    # products and a power of two before them (a value of less than 2^-126 is a
    # multiple of 2^-149, and what that loses is below TINY)
    e = np.abs(y64) * (gamma(8) / 2 + 7 * U32) + G.TINY
    assert np.all(np.abs(G.host(y) - y64) <= e + (np.abs(y64) + e) * G.EPS[dt])
    G.check_mx(q, qs, y64, e)


@pytest.mark.parametrize("dt,cache", [("bf16", "bf16"), ("bf16", "mx"), ("f32", "f32")])
@pytest.mark.parametrize("D", [32, 64, 128, 160, 256])
def test_head_norm_of_values_whose_squares_leave_float32(dt, cache, D):
    rng = np.random.default_rng(D)
    sizes = np.array([1e36, 1e30, 3e19, 1e18, 1.0, 1e-18, 1e-21, 1e-25, 1e-36])
    T, n_q, n_kv, page, rot = len(sizes), 3, 1, 4, D // 2
    x = G.rows(rng, (T, (n_q + 2 * n_kv) * D), "f32")
    x = (x.double() * torch.from_numpy(sizes).cuda()[:, None]).to(G.DT[dt])
    w = [1 + G.rows(rng, (D,), "f32", 0.1) for _ in range(2)]
    pos = np.arange(T)
    freq = (1e4 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)
    k, v, ks, vs = G.empty_cache(rng, 3, n_kv, page, D, dt, cache)
    q = torch.empty((T, n_q, D), dtype=G.DT[dt], device="cuda")
    B.blk_qkv_cache(x, n_q, G.i32(np.arange(T)), k, v, q, positions=G.i32(pos), inv_freq=torch.from_numpy(freq).cuda(),
                    q_norm=w[0], k_norm=w[1], eps=0.0, k_scale=ks, v_scale=vs)
    a = (G.host(x), n_q, n_kv, D, G.host(w[0]), G.host(w[1]), 0.0, pos)
    q64, k64, v64 = O.heads_of(*a, freq)
    for got, ref, plain in ((q, q64, O.heads_of(*a, None)[0]), (k, k64, O.heads_of(*a, None)[1])):
        if ref is k64 and cache == "mx":
            got = O.dequantize_mx8(G.host(k), G.host(ks)).swapaxes(1, 2).reshape(-1, n_kv, D)[:T]
            eps = 2.0 ** -4
        else:
            got = G.host(got) if ref is q64 else G.host(got).swapaxes(1, 2).reshape(-1, n_kv, D)[:T]
            eps = G.EPS[dt]
        # the head norm's bound, and a rotated value is a cos + b sin: |a| + |b|
        # times two products, a sum, the angle and its sine; 8-bit values below
        # the smallest normal one are off by half its step, 2^-10 of the scale,
        # which is at most 2^-7 of the block's largest value
        both = np.abs(plain).copy()
        both[..., :rot // 2] += np.abs(plain[..., rot // 2:rot])
        both[..., rot // 2:rot] += np.abs(plain[..., :rot // 2])
        e = both * (gamma(D + 2) / 2 + (math.pi + 16) * U32) + G.TINY
        low = 2.0 ** -17 * np.max(np.abs(ref), -1, keepdims=True) if eps == 2.0 ** -4 else 0.0
        assert np.all(np.abs(got - ref) <= e + (np.abs(ref) + e) * eps + low)
