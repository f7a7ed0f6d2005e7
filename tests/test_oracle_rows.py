"""Pins of the row operators' float64 oracle: hand-made examples, brute force
and finite differences (CPU)."""

import numpy as np
import pytest

from oracle import rows_ref as ref


def test_sort_by_hand():
    plan = ref.sort_keys_ref([2, 0, 7, 2, -1, 0], 4)
    assert plan["order"].tolist() == [1, 5, 0, 3, 2, 4]
    assert plan["position"].tolist() == [2, 0, 4, 3, 5, 1]
    assert plan["offsets"].tolist() == [0, 2, 2, 4, 4]


def test_sort_by_counting():
    keys = np.random.default_rng(0).integers(-2, 9, 200)
    plan = ref.sort_keys_ref(keys, 7)
    k = np.where((keys >= 0) & (keys < 7), keys, 7)
    for i in range(200):
        assert plan["position"][i] == (k < k[i]).sum() + (k[:i] == k[i]).sum()
        assert plan["order"][plan["position"][i]] == i
    for v in range(8):
        assert plan["offsets"][v] == (k < v).sum()


def test_route_by_hand():
    ln = np.log
    rows = np.array([[ln(1.), ln(3.), ln(3.), ln(1.)], [-np.inf, 5., -np.inf, -np.inf], [-np.inf] * 4])
    w, ids = ref.route_ref(rows, 2, True)
    assert ids.tolist() == [[1, 2], [1, -1], [-1, -1]]
    np.testing.assert_allclose(w, [[.5, .5], [1., 0.], [0., 0.]])
    w, _ = ref.route_ref(rows, 2, False)
    np.testing.assert_allclose(w, [[.375, .375], [1., 0.], [0., 0.]])


@pytest.mark.parametrize("renormalise", [True, False])
def test_route_backward_is_the_derivative(renormalise):
    rng = np.random.default_rng(1)
    logits, g = rng.normal(size=(5, 9)), rng.normal(size=(5, 3))
    logits[0, :7] = -np.inf
    grad = ref.route_backward_ref(g, logits, 3, renormalise)
    h = 1e-5
    for t in range(5):
        for e in range(9):
            up, down = logits.copy(), logits.copy()
            up[t, e] += h
            down[t, e] -= h
            d = ((ref.route_ref(up, 3, renormalise)[0] - ref.route_ref(down, 3, renormalise)[0]) * g).sum() / (2 * h)
            assert abs(d - grad[t, e]) < 1e-8


def test_dispatch_and_combine_invert_each_other():
    rng = np.random.default_rng(2)
    x, ids = rng.normal(size=(20, 5)), rng.integers(0, 6, (20, 3))
    rows, plan = ref.dispatch_ref(x, ids, 6)
    out, _ = ref.combine_ref(rows, np.full((20, 3), 1 / 3), plan)
    np.testing.assert_allclose(out, x)
    for e in range(6):
        for q in range(plan["offsets"][e], plan["offsets"][e + 1]):
            s = plan["order"][q]
            assert ids[s // 3, s % 3] == e
            assert (rows[q] == x[s // 3]).all()


def test_combine_gradients_are_adjoint():
    rng = np.random.default_rng(3)
    ids = rng.integers(-1, 5, (11, 4))
    _, plan = ref.dispatch_ref(rng.normal(size=(11, 3)), ids, 5)
    rows, w, g = rng.normal(size=(44, 3)), rng.normal(size=(11, 4)), rng.normal(size=(11, 3))
    out, _ = ref.combine_ref(rows, w, plan)
    gr, gw, _ = ref.combine_backward_ref(g, rows, w, plan)
    np.testing.assert_allclose((g * out).sum(), (gr * rows).sum())
    np.testing.assert_allclose((g * out).sum(), (gw * w).sum())
    assert (gr[plan["offsets"][-1]:] == 0).all()
    assert (gw.reshape(-1)[(ids.reshape(-1) < 0)] == 0).all()


def test_embed_by_hand_and_adjoint():
    table = np.arange(6.).reshape(3, 2)
    np.testing.assert_array_equal(ref.embed_ref(table, [[2, -1], [0, 3]], 2.),
                                  [[[8, 10], [0, 0]], [[0, 2], [0, 0]]])
    rng = np.random.default_rng(4)
    ids, g, t = rng.integers(-1, 8, 50), rng.normal(size=(50, 3)), rng.normal(size=(7, 3))
    gt, _, count = ref.embed_backward_ref(g, ids, 7, 1.5)
    np.testing.assert_allclose((g * ref.embed_ref(t, ids, 1.5)).sum(), (gt * t).sum())
    assert count.sum() == ((ids >= 0) & (ids < 7)).sum()
