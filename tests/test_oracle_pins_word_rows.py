"""Pins of the oracle of dropout and grouped integers: published generator outputs, counts, worked examples, exact arithmetic."""
import os
from fractions import Fraction

import numpy as np
import pytest

from oracle import word_rows as wr

KAT = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "philox4x32_10_kat.txt")


def test_the_generator_against_its_published_outputs():
    n = 0
    for line in open(KAT):
        words = [w for w in line.split("#")[0].replace(",", " ").split() if len(w) >= 8]
        if len(words) < 10:
            continue
        v = [int(w, 16) for w in words[-10:]]
        got = wr.philox([np.uint64(c) for c in v[:4]], v[4] | v[5] << 32)
        assert [int(x) for x in got] == v[6:10]
        n += 1
    assert n >= 3


def test_bits_depend_on_the_place_alone_and_not_on_the_matrix():
    big = wr.bits(9, 40, 77, 5)
    assert np.array_equal(wr.bits(4, 13, 77, 5), big[:4, :13])
    for other in (wr.bits(9, 40, 78, 5), wr.bits(9, 40, 77, 6), wr.bits(9, 40, 77 + (1 << 40), 5), wr.bits(9, 40, 77, 5 + (1 << 40))):
        assert np.mean(other == big) < 0.01
    assert len(np.unique(big)) > 355                    # 360 draws of 32 bits


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0])
def test_how_many_are_kept(p):
    k = wr.kept(700, 130, p, 1, 2)
    n = k.size
    assert abs(int(k.sum()) - n * (1 - p)) <= 5 * np.sqrt(n * p * (1 - p))
    # neighbours are independent: the joint rate of two places is the product, within five deviations
    for a, b in ((k[:, :-1], k[:, 1:]), (k[:-1], k[1:]), (k[:, :-8], k[:, 8:])):
        q = (1 - p) ** 2
        assert abs(np.mean(a & b) - q) <= 5 * np.sqrt(q * (1 - q) / a.size) + 2 * np.sqrt(p * (1 - p) / n)


def test_a_group_by_hand():
    # least -1, largest 14: b = -1, s = 1
    x = np.array([[-1.0, 14.0, 0.4, 0.5, 0.6, 1.5, 13.49]])
    q, s, b = wr.group_quantize(x, 32)
    assert (s[0, 0], b[0, 0]) == (1.0, -1.0) and list(q[0, :7]) == [0, 15, 1, 2, 2, 2, 14]        # 1.5 and 2.5 codes up: ties to even
    assert np.array_equal(wr.group_numbers(q, s, b, 7)[0], [-1, 14, 0, 1, 1, 1, 13])
    assert np.all(s[0, 1:] == 0) and np.all(b[0, 1:] == 0) and np.all(q[0, 7:] == 0)
    lay = wr.group_layout(q)[0]
    word = int.from_bytes(bytes(lay[:4]), "little")
    assert [(word >> s) & 15 for s in (0, 16, 4, 20, 8, 24, 12, 28)] == [0, 15, 1, 2, 2, 2, 14, 0]


def test_groups_at_the_ends_of_the_range():
    top = float(np.finfo(np.float32).max)
    q, s, b = wr.group_quantize(np.array([[0.0, top]]), 32)
    assert b[0, 0] == 0 and 15 * s[0, 0] <= top and wr.group_numbers(q, s, b, 2)[0, 1] > 0.99 * top
    q, s, b = wr.group_quantize(np.array([[-top, top]]), 32)
    assert b[0, 0] == -wr.BF16_MAX and b[0, 0] + 15 * s[0, 0] <= top
    q, s, b = wr.group_quantize(np.array([[3.0, 3.0], [0.0, 0.0], [2.0 ** -149, 0.0]]), 128)
    assert list(s[:, 0]) == [0, 0, 0] and list(b[:, 0]) == [3, 0, 0]
    q, s, b = wr.group_quantize(np.array([[np.inf, 1.0], [np.nan, 1.0]]), 64)
    assert np.isnan(s[:, 0]).all() and np.isnan(b[:, 0]).all() and not q.any()


def test_rounding_is_to_the_nearest_number_of_the_group_in_exact_arithmetic():
    rng = np.random.default_rng(3)
    x = (rng.normal(size=(3, 96)) * 10.0 ** rng.integers(-6, 6, (3, 96))).astype(np.float32)
    q, s, b = wr.group_quantize(x, 32)
    for i in range(3):
        for k in range(96):
            g = k // 32
            choices = [abs(Fraction(float(x[i, k])) - Fraction(b[i, g]) - c * Fraction(s[i, g])) for c in range(16)]
            assert choices[q[i, k]] == min(choices)
        for g in range(3):
            lo, hi = float(x[i, g * 32:(g + 1) * 32].min()), float(x[i, g * 32:(g + 1) * 32].max())
            assert b[i, g] <= lo and lo - b[i, g] <= 2.0 ** -7 * abs(lo) and abs(s[i, g] * 15 - (hi - b[i, g])) <= 2.0 ** -8 * (hi - b[i, g]) * 1.01


def test_the_gradient_is_the_transpose_of_the_lookup():
    rng = np.random.default_rng(4)
    T, D, t = rng.normal(size=(7, 11)), rng.normal(size=(20, 11)), rng.integers(-1, 8, 20)
    rows = np.where(((t >= 0) & (t < 7))[:, None], T[np.where((t >= 0) & (t < 7), t, 0)], 0.0)
    G, _, _ = wr.embed_dropout_grad(D, t, 7, 0.3, 9, 4, 1.5)
    assert np.allclose((D * wr.dropout(rows, 0.3, 9, 4, 1.5)).sum(), (G * T).sum())


def test_product_of_the_numbers():
    rng = np.random.default_rng(5)
    x, w = rng.normal(size=(3, 70)), rng.normal(size=(4, 70)).astype(np.float32)
    q, s, b = wr.group_quantize(w, 32)
    got, size = wr.group_product(x, q, s, b, 2.0)
    n = wr.group_numbers(q, s, b, 70)
    assert np.allclose(got, [[2.0 * sum(x[i, k] * n[j, k] for k in range(70)) for j in range(4)] for i in range(3)])
    assert np.all(size >= np.abs(got)) and np.abs(n - w).max() <= 0.53 * s.max()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("alpha, beta", [(0.1, 0.01), (0.1, 0.1), (1.0, 0.1), (1.0, 1.0)])
@pytest.mark.parametrize("K", [50, 256])
def test_predictive_weights_of_grouped_models(K, alpha, beta, group):
    """theta as it is, phi in grouped integers.  An element is off by at most s / 2, and the largest of a group by 15 times the rounding of s
    (half a bfloat16 step, 2^-8 s) more; on average the weights are off by what the documents say, 0.6 to 5.3 % of their sum."""
    rng = np.random.default_rng(K)
    theta, phi = rng.dirichlet([alpha] * K, 60), rng.dirichlet([beta] * 200, K).T.copy()
    q, s, b = wr.group_quantize(phi, group)
    numbers = wr.group_numbers(q, s, b, K)
    bound = np.repeat(s, group, axis=1)[:, :K] * (0.5 + 15.0 / 256.0)
    assert np.all(np.abs(numbers - phi) <= 1.000001 * bound + 1e-44)
    want = theta @ phi.T
    far = np.abs(theta @ numbers.T - want)
    assert np.all(far <= 1.000001 * theta @ bound.T + 1e-40)
    assert 0.005 < far.sum() / want.sum() < 0.06


@pytest.mark.parametrize("group", [32, 64, 128])
def test_groups_at_either_end_of_binary32_stand_for_finite_numbers(group):
    """b + 15 s is at most binary32's largest number in magnitude, also where a group lies below the least finite bfloat16 number and s
    is below 0; the reading is within a step of the number, or, of numbers below the least finite bfloat16 number b, at b."""
    top = float(np.finfo(np.float32).max)
    low = -wr.BF16_MAX
    x = np.zeros((6, 128))
    x[0] = -top
    x[1] = np.linspace(-top, low, 128)
    x[2] = (low - top) / 2
    x[3] = top
    x[4] = np.linspace(-low, top, 128)
    x[5, ::2], x[5, 1::2] = -top, top
    x = x.astype(np.float32).astype(np.float64)
    q, step, base = wr.group_quantize(x, group)
    read = wr.group_numbers(q, step, base, 128)
    assert np.all(np.abs(base + 15.0 * step) <= top) and np.all(np.abs(read) <= top)
    assert np.all(step[0] < 0) and np.all(np.abs(read - x) <= np.maximum(np.repeat(np.abs(step), group, axis=1), top + low))
    assert np.all(read[0] == base[0, 0] + 15.0 * step[0, 0])
