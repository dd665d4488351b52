"""The attention half at the ends of the number range and of its precision:
softmax weights that are not rounded to the rows' type, rows without weight
over values that are not finite."""

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
