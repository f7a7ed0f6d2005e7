"""Pins of the logits operators' float64 oracle, and of the expert layer's:
hand-made examples, identities and finite differences (CPU)."""

import numpy as np
import pytest

from oracle import logits_ref as ref
from oracle import rows_ref

LN = np.log


def test_logprobs_by_hand():
    rows = np.array([[LN(1.), LN(2.), LN(1.)], [-np.inf, 3., -np.inf], [-np.inf] * 3, [0., np.nan, 1.]])
    r = ref.logprobs_ref(rows, [1, 0, 2, -1], 2, 1.0)
    np.testing.assert_allclose(r["logprob"], [LN(.5), -np.inf, -np.inf, 0.])
    np.testing.assert_allclose(r["lse"], [LN(4.), 3., -np.inf, np.nan])
    np.testing.assert_allclose(r["entropy"], [1.5 * LN(2.), 0., 0., np.nan])
    assert r["top_ids"].tolist() == [[1, 0], [1, -1], [-1, -1], [2, 0]]
    np.testing.assert_allclose(r["top"], [[LN(.5), LN(.25)], [0., -np.inf], [-np.inf] * 2, [np.nan] * 2])
    # twice the scale squares the odds
    np.testing.assert_allclose(ref.logprobs_ref(rows[:1], [1], 0, 2.0)["logprob"], [LN(4 / 6)])


def test_logprobs_do_not_move_with_the_row():
    rows = np.random.default_rng(0).normal(size=(4, 30))
    a, b = (ref.logprobs_ref(r, [3] * 4, 5, 0.7) for r in (rows, rows + 100))
    for name in ("logprob", "entropy", "top"):
        np.testing.assert_allclose(a[name], b[name], atol=1e-12)
    np.testing.assert_allclose(b["lse"] - a["lse"], 70)


def test_logprobs_of_huge_logits():
    """Rows of one huge value are uniform, as any other constant row."""
    for v in (-3e38, 3e38, 1e300):
        r = ref.logprobs_ref(np.full((1, 4), v), [2], 1, 0.5)
        np.testing.assert_allclose([r["logprob"][0], r["entropy"][0], r["top"][0, 0]], [-LN(4.), LN(4.), -LN(4.)])


def _differences(f, x, h=1e-5):
    grad = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        if x[i] == -np.inf:
            continue
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        grad[i] = (f(up) - f(down)) / (2 * h)
    return grad


def test_logprobs_gradient_is_the_derivative():
    rng = np.random.default_rng(1)
    rows = rng.normal(size=(5, 9)) * 2
    rows[1, 4:] = -np.inf
    ids, scale, k = [2, 1, -1, 9, 0], 1.3, 3
    top_ids = ref.logprobs_ref(rows, ids, k, scale)["top_ids"]
    g = dict(grad_logprob=rng.normal(size=5), grad_lse=rng.normal(size=5), grad_entropy=rng.normal(size=5),
             grad_top=rng.normal(size=(5, k)))

    def total(x):
        r = ref.logprobs_ref(x, ids, k, scale)
        return sum((r[n[5:]] * v).sum() for n, v in g.items())

    got = ref.logprobs_backward_ref(rows, ids, top_ids, scale, **g)
    np.testing.assert_allclose(got, _differences(total, rows), atol=1e-8)
    assert (got[1, 4:] == 0).all()


def test_distill_by_hand():
    rows = np.array([[LN(1.), LN(2.), LN(1.)]] * 4)
    t = LN(np.array([[.5, .25], [.5, .25], [.5, .25], [.5, .25]]))
    ids = [[1, 0], [1, -1], [3, -1], [1, 1]]
    # the teacher's 2/3 and 1/3 against 1/2 and 1/4; one alternative kept; none; the same one twice
    want = [2 / 3 * LN(4 / 3) + 1 / 3 * LN(4 / 3), LN(2.), 0., 2 / 3 * LN(4 / 3) + 1 / 3 * LN(2 / 3)]
    np.testing.assert_allclose(ref.distill_ref(rows, ids, t, 1.0, True), want)
    np.testing.assert_allclose(ref.distill_ref(rows, ids, t, 1.0, False)[:2], [0., 0.], atol=1e-15)


def test_distill_is_least_at_the_teacher():
    """All of a softmax's tokens as alternatives: divergence and gradient are 0 there, and the loss larger elsewhere."""
    rng = np.random.default_rng(2)
    rows = rng.normal(size=(3, 7))
    logp = np.stack([ref.distribution(r, 0.8)[0] for r in rows])
    ids = [list(range(7))] * 3
    for renormalise in (True, False):
        np.testing.assert_allclose(ref.distill_ref(rows, ids, logp, 0.8, renormalise), 0, atol=1e-14)
        np.testing.assert_allclose(ref.distill_backward_ref(np.ones(3), rows, ids, logp, 0.8, renormalise), 0, atol=1e-14)
        assert (ref.distill_ref(rows + rng.normal(size=(3, 7)), ids, logp, 0.8, renormalise) > 1e-3).all()


@pytest.mark.parametrize("renormalise", [True, False])
def test_distill_gradient_is_the_derivative(renormalise):
    rng = np.random.default_rng(3)
    rows = rng.normal(size=(4, 8))
    teacher = np.log(rng.dirichlet(np.ones(8), size=4)[:, :4])
    teacher[0, 1] = -np.inf
    ids = np.array([[1, 2, 3, 4], [0, -1, 7, 8], [5, 5, 5, 1], [-1, -1, 9, 8]])
    g = rng.normal(size=4)
    want = _differences(lambda x: (g * ref.distill_ref(x, ids, teacher, 0.6, renormalise)).sum(), rows)
    np.testing.assert_allclose(ref.distill_backward_ref(g, rows, ids, teacher, 0.6, renormalise), want, atol=1e-8)


def test_expert_layer_by_hand():
    x = np.array([[1., 2.]])
    up = np.array([[[1., 0.], [0., 1.]], [[LN(3.), 0.], [1., 1.]]])  # (E, 2F = 2, C)
    down = np.array([[[1.], [0.]], [[2.], [-1.]]])
    out = rows_ref.expert_layer_ref(x, up, down, [[1.], ], [[1]])[0]
    h = LN(3.) * .75 * 3.  # silu(ln 3) = ln 3 * 3/4
    np.testing.assert_allclose(out, [[2 * h, -h]])
    both = rows_ref.expert_layer_ref(x, up, down, [[.5, 2.]], [[1, 0]])[0]
    np.testing.assert_allclose(both, [[h + 2 * 2 / (1 + np.exp(-1.)), -.5 * h]])
    assert (rows_ref.expert_layer_ref(x, up, down, [[.5, 2.]], [[-1, 2]])[0] == 0).all()


def test_expert_layer_is_dispatch_experts_combine():
    rng = np.random.default_rng(4)
    T, k, E, C, F = 7, 3, 5, 6, 4
    x, up, down = rng.normal(size=(T, C)), rng.normal(size=(E, 2 * F, C)), rng.normal(size=(E, C, F))
    w, ids = rng.normal(size=(T, k)), rng.integers(-1, E, (T, k))
    rows, plan = rows_ref.dispatch_ref(x, ids, E)
    y = np.zeros((T * k, C))
    for e in range(E):
        a, b = plan["offsets"][e], plan["offsets"][e + 1]
        g, v = rows[a:b] @ up[e, :F].T, rows[a:b] @ up[e, F:].T
        y[a:b] = (g / (1 + np.exp(-g)) * v) @ down[e].T
    np.testing.assert_allclose(rows_ref.expert_layer_ref(x, up, down, w, ids)[0], rows_ref.combine_ref(y, w, plan)[0])
