"""The oracle of the attention half of a block, pinned by hand-worked values,
closed forms and invariants."""

import math

import numpy as np
import pytest
import torch

from _util import ROOT  # noqa: F401
from oracle import block as B


def test_e4m3_table_is_the_formats():
    t = torch.arange(128, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(B.E4M3, t)


@pytest.mark.parametrize("most,byte", [(0.0, 0), (448.0, 127), (449.0, 128), (1.75, 119), (1.7500001, 120),
                                       (2.0 ** -130, 0), (math.inf, 255)])
def test_scale_byte(most, byte):
    assert B.scale_byte(most, 448.0) == byte


def test_nearest_even_ties():
    # 0.25 lies between codes 0 and 1, 0.75 between 1 and 2, 5 between 6 and 7 (values 4 and 6)
    assert [B.nearest_even(v, B.E2M1) for v in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, 6.0)] == \
        [0, 2, 2, 4, 4, 6, 6, 7, 7]


def test_quantised_rows_are_within_half_a_step():
    rng = np.random.default_rng(0)
    v = rng.standard_normal((5, 70)) * 2.0 ** rng.integers(-20, 20, (5, 1))
    codes, scales = B.quantize_mx8(v)
    got = B.dequantize_mx8(codes, scales)
    s = np.repeat(B.e8m0(scales), 32, 1)[:, :70]
    assert np.all(np.abs(got - v) <= np.maximum(np.abs(v) * 2.0 ** -4, s * 2.0 ** -10))
    assert np.all(np.abs(v) <= 448 * s) and np.all(np.abs(v).reshape(5, -1).max(1) > 0)


def test_dequantised_w4():
    codes = np.array([[0x10, 0xF8] + [0] * 14], np.uint8)
    v = B.dequantize_w4(codes, np.array([[128]], np.uint8))
    assert v[0, :4].tolist() == [0.0, 1.0, -0.0, -12.0] and not v[0, 4:].any()


def test_rms_of_equal_values():
    h, y = B.rms_norm(np.full((1, 4), 3.0), np.full((1, 4), -1.0), np.array([1.0, 2.0, 3.0, 4.0]), 0.0)
    assert h.tolist() == [[2.0] * 4] and np.allclose(y, [[1, 2, 3, 4]], rtol=1e-15)


def test_rotation_by_a_quarter_turn():
    v = np.array([[[1.0, 2.0, 5.0]]])
    r = B.rotate(v, [1], [math.pi / 2])
    assert np.allclose(r, [[[-2.0, 1.0, 5.0]]])


def test_kv_extend_by_hand():
    # pages of 4; sequence 0 holds 5 tokens (pages 7, 2), 1 is finished (3 tokens, page 5), 2 is new
    table = np.array([[7, 2, -1], [5, -1, -1], [-1, -1, -1]], np.int32)
    free = np.array([0, 1, 3, 4, 6, 9, 9, 9], np.int32)
    r = B.kv_extend([5, 3, 0], [4, -1, 2], 5, table, free, 4, 8)
    # the stack is 0 1 3 4 6 and then 5; sequence 0 takes 5, sequence 2 takes 6
    assert r["block_table"].tolist() == [[7, 2, 5], [5, -1, -1], [6, -1, -1]]
    assert r["free_pages"].tolist() == [0, 1, 3, 4, 6, 5, 9, 9] and r["n_free_out"].tolist() == [4]
    assert r["len_out"].tolist() == [9, 0, 2] and r["row_offsets"].tolist() == [0, 4, 4, 6]
    # positions 5, 6, 7 in page 2, 8 in page 5, then 0, 1 in page 6
    assert r["slot_map"].tolist() == [9, 10, 11, 20, 24, 25, -1, -1] and r["positions"].tolist() == [5, 6, 7, 8, 0, 1, 0, 0]
    assert r["status"].tolist() == [6, 2, 0, 1] and r["accepted"].tolist() == [1, 1, 1]


def test_kv_extend_refuses_what_does_not_fit():
    table = np.full((4, 2), -1, np.int32)
    free = np.arange(3, dtype=np.int32)
    # 0: too long for its table; 1: two pages; 2: two more than there are; 3: nothing to take
    r = B.kv_extend([0, 0, 0, 1], [9, 8, 8, 1], 3, table, free, 4, 64)
    assert r["accepted"].tolist() == [0, 1, 0, 1] and r["status"].tolist() == [26, 2, 2, 0]
    assert r["len_out"].tolist() == [0, 8, 0, 2] and r["n_free_out"].tolist() == [1]
    # sequence 3's page entry is none: no slot
    assert r["slot_map"][25] == -1 and (r["slot_map"][:9] == -1).all() and (r["slot_map"][9:17] >= 0).all()


def test_keys_on_pages_that_are_none_are_left_out():
    cache = np.arange(2 * 1 * 2 * 1, dtype=float).reshape(2, 1, 2, 1)
    assert B.keys_of(cache, [1, -1, 0], 5, 2)[0, :, 0].tolist() == [2.0, 3.0, 0.0]
    assert B.keys_of(cache, [2], 2, 2).shape == (1, 0, 1)


def test_attention_closed_forms():
    rng = np.random.default_rng(1)
    q, v = rng.standard_normal((4, 8)), rng.standard_normal((2, 5, 8))
    out, w = B.attention(q, np.zeros((2, 5, 8)), v, 1.0)
    assert np.allclose(out, np.repeat(v.mean(1), 2, 0)) and np.allclose(w, 0.2)
    assert not B.attention(q, np.zeros((2, 0, 8)), np.zeros((2, 0, 8)), 1.0)[0].any()
