"""Row operators on the GPU where their rules change over: sizes on both sides
of each variant's border, plans and gradients in the forms that a caller may
give them.  Tolerances as in test_gpu_rows.py, or derived beside the test.
"""

import numpy as np
import pytest
import torch

import test_gpu_rows as plain
from _gpu import DEV, say
from oracle import rows_ref as ref
from paper_2211_17111_amd import rows
from test_gpu_rows import BF16, F16, F32, TYPES, U, _half_step, _ids, _near, _normal, _np, _same_plan

pytestmark = pytest.mark.gpu


def test_counts_past_32_bits_are_refused():
    """The library takes experts and choices as 32-bit integers: larger ones must not arrive as their low bits."""
    wide = (1 << 32) + 5
    x, empty = _normal(3, 16), torch.empty((0, wide), dtype=F16, device=DEV)
    w, ids = torch.empty((0, 2), device=DEV), torch.empty((0, 2), dtype=torch.int32, device=DEV)
    many_w, many_ids = torch.empty((0, wide), device=DEV), torch.empty((0, wide), dtype=torch.int32, device=DEV)
    for f in (lambda: rows.route_forward(empty, 2), lambda: rows.route_forward(x[:0], wide),
              lambda: rows.route_forward(x, wide), lambda: rows.route_backward(w, empty, w, ids),
              lambda: rows.route_backward(many_w, x[:0], many_w, many_ids)):
        with pytest.raises(ValueError):
            f()


# --------------------------------------------------------------------- plans

def test_order_of_a_matrix_of_ids():
    """sort_keys takes any shape: its plan serves one slot to a token and rows of slots alike."""
    B, S, E, C = 7, 5, 6, 24
    keys = _ids(B, S, E, 4)
    ids = torch.from_numpy(keys).to(DEV)
    plan = rows.sort_keys(ids, E)
    for T, k in ((B * S, 1), (B, S)):
        x, g, w = _normal(T, C, seed=1), _normal(T * k, C, seed=2), _normal(T, k, seed=3)
        got, same = rows.dispatch_forward(x, plan)
        want, wplan = ref.dispatch_ref(_np(x), keys.reshape(T, k), E)
        assert same is plan and np.array_equal(_np(got), want)
        _same_plan(plan, wplan)
        want, mag = ref.combine_ref(_np(g), np.ones((T, k)), wplan)
        _near(rows.dispatch_backward(g, plan, k), want, (k + 2) * U * mag + _half_step(want, F32), f"k={k}")
        want, mag = ref.combine_ref(_np(g), _np(w), wplan)
        _near(rows.combine_forward(g, w, plan), want, (k + 2) * U * mag + _half_step(want, F32), f"combine k={k}")
        leaf = x.clone().requires_grad_()
        rows.dispatch(leaf, plan)[0].backward(g)
        assert torch.equal(leaf.grad, rows.dispatch_backward(g, plan, k))


@pytest.mark.parametrize("renormalise", [True, False])
def test_route_gradient_of_ids_outside(renormalise):
    """An id that names no expert has no gradient, whichever side it lies on."""
    T, E, k = 21, 20, 4
    logits, g = plain._logits(T, E, F32, 1), _normal(T, k, seed=2)
    w, ids = rows.route_forward(logits, k, renormalise)
    outside = torch.rand((T, k), generator=torch.Generator().manual_seed(3)).to(DEV) < 0.4
    outside[0], outside[1] = True, False
    want = rows.route_backward(g, logits, w, torch.where(outside, -1, ids).int(), renormalise)
    for v in (E, E + 9, (1 << 31) - 1, -(1 << 31)):
        got = rows.route_backward(g, logits, w, torch.where(outside, v, ids).int(), renormalise)
        assert torch.equal(got, want), v


# ------------------------------------------------------ what gradients keep

def test_route_keeps_no_logits_that_its_gradient_does_not_read():
    logits, g = plain._logits(9, 20, BF16, 1), _normal(9, 4, seed=2)
    for renormalise in (True, False):
        leaf = logits.clone().requires_grad_()
        l = leaf * 1
        w, ids = rows.route(l, 4, renormalise)
        want = rows.route_backward(g, logits, w.detach(), ids, renormalise)
        w.backward(g, retain_graph=True)
        assert leaf.grad.dtype == BF16 and torch.equal(leaf.grad, want)
        with torch.no_grad():
            l.zero_()  # (the buffer is used again)
        if renormalise:
            leaf.grad = None
            w.backward(g)
            assert torch.equal(leaf.grad, want)
        else:  # the softmax over all experts is formed again from them
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                w.backward(g)


def test_combine_keeps_no_operand_that_its_gradients_do_not_read():
    T, k, E, C = 13, 3, 5, 40
    _, plan = rows.dispatch_forward(_normal(T, C), torch.from_numpy(_ids(T, k, E, 1)).to(DEV), E)
    y0, w0, g = _normal(T * k, C, dtype=BF16, seed=1), _normal(T, k, seed=2), _normal(T, C, dtype=BF16, seed=3)
    want = rows.combine_backward(g, y0, w0, plan)
    for on in ((True, False), (False, True), (True, True)):
        leaves = [t.clone().requires_grad_(r) for t, r in zip((y0, w0), on)]
        used = [t * 1 for t in leaves]
        out = rows.combine(*used, plan)
        out.backward(g, retain_graph=True)
        for t, r, v in zip(leaves, on, want):
            assert (t.grad is None) == (not r)
            if r:
                assert t.grad.dtype == t.dtype and torch.equal(t.grad, v)
                one, = torch.autograd.grad(out, t, g, retain_graph=True)
                assert torch.equal(one, v)
        with torch.no_grad():
            for t, r in zip(used, on):
                if r:
                    t.zero_()  # (the operand whose own gradient is wanted is not read for it)
        if on == (True, True):
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                out.backward(g)
            continue
        for t in leaves:
            t.grad = None
        out.backward(g)
        for t, r, v in zip(leaves, on, want):
            assert not r or torch.equal(t.grad, v)
