"""Pins of the word-table oracle: known roundings, closed forms, differences and identities.  CPU only."""
import numpy as np
import pytest

from oracle import word_tables as wt


def one(values):
    codes, scales = wt.quantize(np.array([values], np.float64))
    return wt.numbers(codes, scales, len(values))[0], scales[0]


def test_every_representable_number_is_kept():
    for e in (-127, -126, -3, 0, 1, 40, 125):
        v = np.concatenate((wt.SIZES, -wt.SIZES)) * 2.0 ** e
        got, scales = one(v)
        assert np.array_equal(got, v) and scales[0] == e + 127


@pytest.mark.parametrize("x, want", [(0.25, 0.0), (0.26, 0.5), (0.75, 1.0), (0.74, 0.5), (1.25, 1.0), (1.75, 2.0), (2.5, 2.0), (2.51, 3.0), (3.5, 4.0),
                                     (5.0, 4.0), (5.01, 6.0), (6.9, 6.0), (7.99, 6.0)])
def test_nearest_and_ties(x, want):
    got, scales = one([4.0, x, -x])                       # 4 .. 7.99: the block's power of two is 1
    assert scales[0] == 127 and got[1] == want and got[2] == -want


def test_block_borders_padding_and_bad_blocks():
    x = np.zeros((1, 70))
    x[0, 31], x[0, 32], x[0, 65] = 6.0, 0.375, np.inf
    codes, scales = wt.quantize(x)
    assert codes.shape == (1, 64) and scales.tolist() == [[127, 123, 255, 0]]
    v = wt.numbers(codes, scales, 70)[0]
    assert v[31] == 6.0 and v[32] == 0.375 and np.all(np.isnan(v[64:])) and not np.any(np.isnan(v[:64]))
    assert one([2.0 ** -149, 0.0])[0].tolist() == [0.0, 0.0]
    assert one([0.0] * 5)[1].tolist() == [0, 0, 0, 0]


def test_gradient_is_the_transpose_of_the_lookup_and_matches_differences():
    rng = np.random.default_rng(1)
    tokens = np.array([3, 0, -1, 3, 7, 3, 1 << 33, 6])
    table, w = rng.normal(size=(7, 5)), rng.normal(size=(8, 5))
    out = wt.embed(table, tokens, 1.5)
    assert np.all(out[[2, 4, 6]] == 0.0)
    g, size, terms = wt.embed_grad(w, tokens, 7, 1.5)
    d = rng.normal(size=table.shape)
    assert np.isclose((wt.embed(d, tokens, 1.5) * w).sum(), (d * g).sum(), rtol=1e-12)
    h = 0.125                                              # the lookup is linear: the difference quotient is exact to rounding
    for r in range(7):
        for c in range(5):
            up = table.copy()
            up[r, c] += h
            assert np.isclose(((wt.embed(up, tokens, 1.5) - out) * w).sum() / h, g[r, c], atol=1e-12)
    assert terms.tolist() == [1, 0, 0, 3, 0, 0, 1] and np.all(size >= np.abs(g) - 1e-15)


def test_product_of_small_integers():
    a, b = np.array([[1.0, -2.0, 3.0]]), np.array([[4.0, 0.5, 6.0], [0.0, 1.0, 0.0]])
    y, size = wt.product(a, b, 2.0)
    assert y.tolist() == [[42.0, -4.0]] and size.tolist() == [[46.0, 4.0]]
