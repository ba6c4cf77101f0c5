"""Pins of the 4-bit oracle: the format's table, rounding by hand and by brute force, scales of
exact powers, subnormal and special blocks, and planted mistakes."""
import numpy as np
import pytest

from oracle import mx4


def test_e2m1_table():
    assert mx4.GRID.tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]


def block(*v):
    x = np.zeros((1, 32))
    x[0, :len(v)] = v
    return x


@pytest.mark.parametrize("x,code", [
    (0.25, 0), (0.2500001, 1), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (4.999, 6), (5.0, 6), (5.001, 7),
    (6.9, 7), (7.999, 7), (-0.25, 8), (-0.75, 10), (-5.0, 14), (-0.0, 8)])
def test_rounding_by_hand(x, code):
    c, s = mx4.quantise(block(4.0, x))          # the largest magnitude is in [4, 8): scale 1
    assert s[0, 0] == 127 and c[0, 1] == code and c[0, 0] == 6


def test_rounding_is_to_the_nearest():
    x = np.linspace(-7.99, 7.99, 32 * 4001).reshape(-1, 32)
    x[:, 0] = 4.0
    c, s = mx4.quantise(x)
    assert (s == 127).all()
    best = np.abs(np.clip(x, -6, 6)[..., None] - mx4.GRID).min(axis=-1)
    assert (np.abs(np.clip(x, -6, 6) - mx4.values(c, s)) == best).all()


@pytest.mark.parametrize("top,scale", [(1.0, 125), (1.999, 125), (2.0, 126), (4.0, 127), (2.0 ** 127, 252), (3e38, 252),
                                       (2.0 ** -125, 0), (2.0 ** -124, 1), (2.0 ** -140, 0), (0.0, 0),
                                       (np.inf, 255), (np.nan, 255)])
def test_scales(top, scale):
    assert mx4.quantise(block(top))[1][0, 0] == scale
    assert mx4.quantise(block(0.0, -top))[1][0, 0] == scale


def test_special_blocks_are_nan_and_neighbours_are_not():
    x = np.ones((1, 96))
    x[0, 40] = np.inf
    v = mx4.values(*mx4.quantise(x))
    assert np.isnan(v[0, 32:64]).all() and (v[0, :32] == 1).all() and (v[0, 64:] == 1).all()


def test_pack_round_trip():
    c = np.arange(64, dtype=np.uint8).reshape(2, 32) % 16
    p = mx4.pack(c)
    assert p.shape == (2, 16) and p[0, 0] == 0x10 and (mx4.unpack(p) == c).all()


def test_sort_by_hand():
    ids = np.array([[1, 0], [1, -1], [2, 1], [9, 0]])
    offsets, order, pos = mx4.sort_slots(ids, 3, 2, 11)
    assert offsets.tolist() == [0, 2, 6, 8]
    assert order.tolist() == [1, 7, 0, 2, 5, -1, 4, -1, -1, -1, -1]
    assert pos.tolist() == [2, 0, 3, -1, 6, 4, -1, 1]


def test_planted_mistakes_are_seen():
    x = np.linspace(-7.9, 7.9, 320).reshape(10, 32)
    x[:, 0] = 4.0
    c, s = mx4.quantise(x)
    assert (np.minimum(np.round(np.abs(x) * 2) / 2, 6) != np.abs(mx4.values(c, s))).any()      # a fixed step
    assert (mx4.values(c, s - 1) != mx4.values(c, s)).any()                                    # a scale off by one
    assert (mx4.unpack(mx4.pack(c))[:, ::-1] != c).any()
