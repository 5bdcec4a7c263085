"""Pins of oracle/b128.py: hand-worked cases, textbook special cases, brute force (no GPU)."""
import itertools
import math

import numpy as np
import pytest

from oracle import b128, quant_e4m3


def test_select_by_hand():
    # sigmoid(0) = 1/2, sigmoid(ln 3) = 3/4, sigmoid(-ln 3) = 1/4
    l = np.array([[0.0, math.log(3), -math.log(3), 0.0]])
    idx, w = b128.select(l, 2)
    assert idx.tolist() == [[1, 0]] and np.allclose(w, [[0.6, 0.4]])
    idx, w = b128.select(l, 2, bias=[0, 0, 0.6, 0.0], renormalize=False, scale=2.0)  # keys 1/2, 3/4, 0.85, 1/2: the bias is not in the weights
    assert idx.tolist() == [[2, 1]] and np.allclose(w, [[0.5, 1.5]])
    # groups {0, 1} and {2, 3}: by their best 3/4 against 1/2, by their two best 5/4 against 3/4
    assert b128.select(l, 1, n_groups=2, groups_kept=1, group_top=1)[0].tolist() == [[1]]
    l = np.array([[3.0, -9.0, 2.0, 2.0]])
    assert b128.select(l, 1, n_groups=2, groups_kept=1, group_top=1)[0].tolist() == [[0]]
    assert b128.select(l, 1, n_groups=2, groups_kept=1, group_top=2)[0].tolist() == [[2]]


def test_select_softmax_is_the_whole_rows():
    rng = np.random.default_rng(0)
    l = rng.standard_normal((20, 12))
    p = np.exp(l) / np.exp(l).sum(1, keepdims=True)
    idx, w = b128.select(l, 12, score="softmax", renormalize=False)
    assert np.array_equal(idx, np.argsort(-l, 1, kind="stable"))
    assert np.allclose(w, np.take_along_axis(p, idx.astype(int), 1), rtol=1e-14)
    _, w = b128.select(l, 3, score="softmax", scale=2.5)
    assert np.allclose(w.sum(1), 2.5)


def test_select_by_brute_force():
    """The chosen set is the best of all subsets that lie in the best of all sets of groups."""
    rng = np.random.default_rng(1)
    for _ in range(60):
        l, bias = rng.standard_normal((1, 8)), rng.standard_normal(8) * 0.3
        s = 1 / (1 + np.exp(-l[0]))
        key = s + bias
        idx, _ = b128.select(l, 2, bias=bias, n_groups=4, groups_kept=2, group_top=2)
        groups = max(itertools.combinations(range(4), 2), key=lambda c: sum(key[2 * g] + key[2 * g + 1] for g in c))
        best = max(itertools.combinations([e for g in groups for e in (2 * g, 2 * g + 1)], 2), key=lambda c: key[list(c)].sum())
        assert set(idx[0].tolist()) == set(best)


def test_select_without_keys():
    inf, nan = math.inf, math.nan
    idx, w = b128.select([[-inf, 1.0, nan, -inf]], 3)
    assert idx.tolist() == [[1, 0, 2]] and w.tolist() == [[1.0, 0.0, 0.0]]
    idx, w = b128.select([[-inf] * 4], 2, score="softmax")
    assert idx.tolist() == [[0, 1]] and w.tolist() == [[0.0, 0.0]]
    idx, w = b128.select([[inf, 0.0, inf, 5.0]], 3, score="softmax", renormalize=False)
    assert idx.tolist() == [[0, 2, 1]] and w.tolist() == [[0.5, 0.5, 0.0]]
    idx, w = b128.select([[0.0, 0.0, 0.0, 0.0]], 2, bias=[-inf, 0.0, nan, 0.0])
    assert idx.tolist() == [[1, 3]]
    # a group with one key and one without is worth that key; a negative sum is less than it
    idx, _ = b128.select([[0.0, -inf, 0.0, 0.0]], 1, bias=[0.0, 0.0, -0.9, -0.2], n_groups=2, groups_kept=1, group_top=2)
    assert idx.tolist() == [[0]]
    # equal keys: the lower index, equal groups: the lower group
    assert b128.select(np.zeros((1, 8)), 2, n_groups=4, groups_kept=2)[0].tolist() == [[0, 1]]


def test_e4m3_is_the_nearest_of_all_numbers():
    numbers = np.array(sorted({v for v in quant_e4m3.code_values() if not math.isnan(v)}))
    rng = np.random.default_rng(2)
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.standard_normal(4000) * 0.02, numbers, (numbers[1:] + numbers[:-1]) / 2])
    got = b128.e4m3(x)
    assert np.isin(got, numbers).all()
    distance = np.abs(numbers[None] - x[:, None]).min(1)
    assert np.array_equal(np.abs(got - x), distance)
    mid = (numbers[1:] + numbers[:-1]) / 2  # a tie goes to the number whose last bit is 0: every second one
    order = np.searchsorted(numbers, b128.e4m3(mid[mid > 0]))
    zero = np.searchsorted(numbers, 0.0)
    assert ((order - zero) % 2 == 0).all()


def test_scale_and_quantize():
    assert b128.scale_exponent(448.0) == 0 and b128.scale_exponent(448.1) == 1 and b128.scale_exponent(224.0) == -1
    assert b128.scale_exponent(0.0) == 0 and b128.scale_exponent(1e-40) == -126 and b128.scale_exponent(3.4e38) == 120
    x = np.zeros((3, 300))
    x[0, 0], x[0, 130], x[1, 299], x[2, 5], x[2, 6] = 448.0, 900.0, -1.0, math.inf, 3.0
    number, scale = b128.quantize(x)
    assert scale.tolist() == [[127, 129, 127, 127], [127, 127, 119, 127], [120, 127, 127, 127]]
    assert number[0, 130] == 224.0 and b128.value(number, scale)[0, 130] == 896.0  # 225 lies between 224 and 240
    assert number[1, 299] == -256.0 and math.isnan(number[2, 5]) and number[2, 6] == 384.0
    number, scale = b128.quantize(np.full((200, 16), 7.0), 128)
    assert scale.shape == (2, 4) and scale[0, 0] == 121 and (b128.value(number, scale, 128) == 7.0).all()


@pytest.mark.parametrize("activation", ["relu", "silu"])
def test_ffn_of_numbers_that_e4m3_holds(activation):
    """Small whole numbers and a hidden row that e4m3 holds: the result is the plain one."""
    rng = np.random.default_rng(3)
    x = rng.integers(-2, 3, (6, 16)).astype(float)
    w2 = rng.integers(-2, 3, (2, 16, 16)).astype(float)
    eye = np.stack([np.eye(16)] * 2)
    offsets = [0, 4, 6]
    if activation == "relu":
        y, bound = b128.ffn(x, eye, w2, offsets, "relu")
        want = np.maximum(x, 0)
    else:
        big = np.zeros((2, 2, 16, 16))  # silu(64 x) = 64 x for x >= 1, u = x: h = 64 x^2 there
        big[:, 0], big[:, 1] = 64 * eye, eye
        y, bound = b128.ffn(np.abs(x), big, w2, offsets, "silu")
        want = 64 * x * x
    want = np.concatenate([want[:4] @ w2[0].T, want[4:] @ w2[1].T])
    assert np.allclose(y, want, atol=1e-9) and (bound >= 0).all() and bound.max() < 1e-3 * np.abs(want).max() + 1e-9


def test_ffn_bound_holds_for_planted_errors():
    """Sums that are off by as much as allowed move the result by no more than the bound."""
    rng = np.random.default_rng(4)
    x, w1, w2 = rng.standard_normal((5, 32)), rng.standard_normal((1, 2, 48, 32)), rng.standard_normal((1, 32, 48))
    for error in (1e-6, 1e-3):
        y, bound = b128.ffn(x, w1, w2, [0, 5], "silu", sum_error=error)
        g, gs = b128.gemm(x, w1[:, 0], [0, 5])
        u, us = b128.gemm(x, w1[:, 1], [0, 5])
        for _ in range(20):
            a, b = g + error * gs * rng.uniform(-1, 1, g.shape), u + error * us * rng.uniform(-1, 1, u.shape)
            q = b128.value(*b128.quantize(a / (1 + np.exp(-a)) * b))
            assert (np.abs(q @ w2[0].T - y) <= bound + 1e-12).all()
