"""Pins of the 4-bit cache's oracle: hand-computed roundings, the layout's
positions, and block tables written out by hand."""
import numpy as np
import pytest

from oracle import block_tables, kv4_read, kv4_round, kv4_values
from oracle.kv4 import kv4_write, nibble_at, scale_at


def _block(*values):
    x = np.zeros(32)
    x[:len(values)] = values
    return x


def test_roundings_by_hand():
    # the largest is 7: scale 1, ties at .25, .75, 1.25, 1.75, 2.5, 3.5, 5 go to the even code
    x = _block(7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.3, -0.0, -6.9, 0.24)
    codes, scales = kv4_round(x)
    assert scales.tolist() == [127]
    assert codes[:12].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 9, 8, 15, 0]
    # just above 7 the scale doubles
    codes, scales = kv4_round(_block(7.0 + 2 ** -5, 1.0))
    assert scales.tolist() == [128] and codes[:2].tolist() == [6, 1]
    assert kv4_values(codes, scales)[:2].tolist() == [8.0, 1.0]


def test_extremes():
    codes, scales = kv4_round(np.zeros(32))
    assert scales.tolist() == [2] and not codes.any()
    codes, scales = kv4_round(_block(np.inf, -np.inf, np.nan, 1.0, 3e38))
    assert scales.tolist() == [252] and codes[:5].tolist() == [7, 15, 0, 0, 7]
    assert np.isfinite(kv4_values(codes, scales)).all()
    codes, scales = kv4_round(_block(2.0 ** -126, 2.0 ** -127, 2.0 ** -130))
    assert scales.tolist() == [2] and codes[:3].tolist() == [1, 0, 0]


@pytest.mark.parametrize("seed", range(5))
def test_no_value_is_off_by_more_than_half_a_step(seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((50, 64)) * np.exp(rng.uniform(-20, 20, (50, 1)))
    codes, scales = kv4_round(x)
    got = kv4_values(codes, scales)
    unit = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)
    step = np.where(np.abs(x) < 2 * unit, 0.5, np.where(np.abs(x) < 4 * unit, 1.0, 2.0)) * unit
    assert (np.abs(got - x) <= step / 2).all()
    top = np.abs(x).reshape(50, 2, 32).max(-1)
    assert (top <= 7 * unit[:, ::32]).all() and (top > 3.5 * unit[:, ::32]).all()


@pytest.mark.parametrize("d", [64, 128])
def test_records_hold_every_key_and_dim_once(d):
    for which in "kv":
        assert sorted(nibble_at(which, d).ravel().tolist()) == list(range(16 * d))
    assert sorted(scale_at(d).ravel().tolist()) == list(range(8 * d, 17 * d // 2))
    # by hand: key 5, dim 37 of d = 128: K piece 1 (dims 32-63), byte 5 * 16 + 16 * 16 + 2, high half
    if d == 128:
        assert nibble_at("k", d)[5, 37] == 2 * (16 * 16 + 5 * 16 + 2) + 1
        assert nibble_at("v", d)[5, 37] == 2 * (((1 * 16 + 4) * 4 + 1) * 4 + 2) + 1
        assert scale_at(d)[5, 1] == 1024 + 16 + 5


@pytest.mark.parametrize("d", [64, 128])
def test_write_then_read(d):
    rng = np.random.default_rng(1)
    pages = rng.integers(0, 256, (3, 2, 17 * d // 2)).astype(np.uint8)
    codes, scales = kv4_round(rng.standard_normal((2, d)))
    for which in "kv":
        before = kv4_read(which, pages, d)
        new = pages.copy()
        kv4_write(which, new, 1, 9, codes, scales)
        after = kv4_read(which, new, d)
        assert np.array_equal(after[0][1, 9], codes) and np.array_equal(after[1][1, 9], scales)
        for x, y in zip(before, after):
            x[1, 9] = y[1, 9]
            assert np.array_equal(x, y)


def test_block_tables_by_hand():
    # 14 cached + 4 new tokens (one new page), 16 + 1 (one), 3 + 2 (none), 0 + 33 (three)
    seqs = [[4, 18, 0], [1, 17, 4], [2, 5, 5], [33, 33, 7]]
    table = np.full((4, 3), -1)
    table[0, 0], table[1, 0], table[2, 0] = 9, 8, 7
    got, slots, taken = block_tables(seqs, [5, 4, 3, 2, 1, 0], table, 10)
    assert got.tolist() == [[9, 5, -1], [8, 4, -1], [7, -1, -1], [3, 2, 1]] and taken == 5
    assert [slots[i] for i in range(8)] == [9 * 16 + 14, 9 * 16 + 15, 5 * 16, 5 * 16 + 1, 4 * 16, 7 * 16 + 3,
                                            7 * 16 + 4, 3 * 16]
    assert slots[39] == 16
