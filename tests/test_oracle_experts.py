"""Pins of the experts' oracle: closed forms, other formulations, brute force."""
import itertools

import numpy as np
import pytest
import torch

from oracle import experts as ox


def test_scores_are_torch_softmax_and_sigmoid():
    l = np.random.default_rng(0).standard_normal(37) * 5
    t = torch.from_numpy(l)
    np.testing.assert_allclose(ox.scores(l, False), torch.softmax(t, 0).numpy(), rtol=1e-13)
    np.testing.assert_allclose(ox.scores(l, True), torch.sigmoid(t).numpy(), rtol=1e-13)
    assert ox.scores(np.array([-200.0, -80.0]), True).tolist() == [1 / (1 + np.exp(80.0))] * 2


@pytest.mark.parametrize("renorm", [False, True])
def test_plain_choice_is_torch_topk(renorm):
    rng = np.random.default_rng(1)
    for _ in range(20):
        l = rng.standard_normal(16)
        e, w = ox.choose(l, 5, renorm=renorm, scale=2.0)
        p, i = torch.softmax(torch.from_numpy(l), 0).topk(5)
        assert e.tolist() == i.tolist()
        np.testing.assert_allclose(w, 2 * (p / p.sum() if renorm else p).numpy(), rtol=1e-12)


def test_the_bias_moves_the_choice_and_not_the_weight():
    l = np.array([0.0, 1.0, 2.0, 3.0])
    e, w = ox.choose(l, 2, sigmoid=True, bias=np.array([5.0, 0, 0, 0]), renorm=False)
    assert e.tolist() == [0, 3]
    np.testing.assert_allclose(w, 1 / (1 + np.exp(-l[[0, 3]])))


def test_the_choice_is_the_best_of_all():
    """Among all sets of two groups and all triples in them, the one of the largest values."""
    rng = np.random.default_rng(2)
    for _ in range(10):
        l, b = rng.standard_normal(12), rng.standard_normal(12) * 0.3
        v = ox.scores(l, True) + b
        best = max(itertools.combinations(range(4), 2),
                   key=lambda gs: sum(max(v[i] + v[j] for i, j in itertools.combinations(range(3 * g, 3 * g + 3), 2)) for g in gs))
        triple = max(itertools.combinations([e for e in range(12) if e // 3 in best], 3), key=lambda c: sum(v[list(c)]))
        assert sorted(ox.choose(l, 3, sigmoid=True, bias=b, groups=4, top_groups=2)[0]) == sorted(triple)


def test_ties_and_ruled_out():
    inf = np.inf
    assert ox.choose(np.zeros(6), 3)[0].tolist() == [0, 1, 2]
    e, w = ox.choose(np.array([-inf, 1.0, np.nan, 1.0]), 3)
    assert e.tolist() == [1, 3, -1] and w.tolist() == [0.5, 0.5, 0.0]
    assert ox.choose(np.full(4, -inf), 2)[0].tolist() == [-1, -1]
    assert ox.choose(np.array([0.0, inf, 3e38]), 2)[0].tolist() == [1, 2]
    # a group whose experts are ruled out is never kept before one that has any
    assert ox.choose(np.array([-inf, -inf, -5.0, -inf]), 1, groups=2, top_groups=1)[0].tolist() == [2]


def test_grouping_is_a_stable_sort():
    rng = np.random.default_rng(3)
    expert = rng.integers(-1, 5, (20, 3))
    offsets, order, place = ox.group(expert, 5)
    flat = expert.reshape(-1)
    live = np.flatnonzero(flat >= 0)
    want = live[np.argsort(flat[live], kind="stable")]
    assert order[:len(want)].tolist() == want.tolist() and (order[len(want):] == -1).all()
    assert (place.reshape(-1)[want] == np.arange(len(want))).all() and (place[expert < 0] == -1).all()
    assert offsets[-1] == len(want) and (flat[order[:len(want)]] == ox.expert_of(offsets)).all()


def test_combine_is_a_matrix_product():
    rng = np.random.default_rng(4)
    y, w, place = rng.standard_normal((12, 7)), rng.random((4, 3)), rng.permutation(12).reshape(4, 3)
    place[1, 2] = -1
    m = np.zeros((4, 12))
    for t, j in itertools.product(range(4), range(3)):
        if place[t, j] >= 0:
            m[t, place[t, j]] = w[t, j]
    add = rng.standard_normal((4, 7))
    np.testing.assert_allclose(ox.combine(y, w, place, add), m @ y + add, rtol=1e-13)


def test_block_of_one_expert_is_the_dense_block():
    rng = np.random.default_rng(5)
    x, g, u, d = rng.standard_normal((3, 8)), rng.standard_normal((1, 6, 8)), rng.standard_normal((1, 6, 8)), rng.standard_normal((1, 4, 6))
    a, b = torch.from_numpy(x @ g[0].T), torch.from_numpy(x @ u[0].T)
    want = (torch.nn.functional.silu(a) * b).numpy() @ d[0].T
    np.testing.assert_allclose(ox.block(x, np.zeros((3, 1)), g, u, d, top_k=1), want, rtol=1e-12)
