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


def _all_forms(x, w_logits, y, w, table, ids, tids, plan, E, k):
    """Every differentiable form, the router in both."""
    return [rows.route(w_logits, k)[0], rows.route(w_logits, k, False)[0], rows.dispatch(x, ids, E)[0],
            rows.dispatch(x, plan)[0], rows.combine(y, w, plan), rows.embed(table, tids, 2.0)]


def test_gradients_of_operands_that_hooks_moved_or_changed():
    """What a gradient keeps may come back through hooks: from the host it is used, in another type or shape refused."""
    T, k, E, C, V = 11, 3, 6, 20, 15
    ids, tids = torch.from_numpy(_ids(T, k, E, 1)).to(DEV), torch.from_numpy(plain._keys(T, V, 2)).to(DEV)
    _, plan = rows.dispatch_forward(_normal(T, C), ids, E)
    shapes = [(T, C), (T, E), (T * k, C), (T, k), (V, C)]
    x, l, y, w, table = [_normal(*s, seed=i).requires_grad_() for i, s in enumerate(shapes)]

    def grads():
        leaves = (x, l, y, w, table)
        for t in leaves:
            t.grad = None
        outs = _all_forms(x, l, y, w, table, ids, tids, plan, E, k)
        return outs, lambda: (sum((o * o).sum() for o in outs).backward(), [t.grad for t in leaves])[1]

    want = grads()[1]()
    with torch.autograd.graph.save_on_cpu():
        _, back = grads()
        got = back()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for change in (lambda t: t.half() if t.is_floating_point() else t.short(), lambda t: t[:1] if t.dim() == 2 else t[:4]):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, change):
            outs, _ = grads()
        for o in outs:
            with pytest.raises(ValueError):
                torch.autograd.backward(o, torch.ones_like(o))


# -------------------------------------------------------------------- router

@pytest.mark.parametrize("E,k", [(2, 2), (16, 2), (64, 4), (256, 12), (300, 3)])
def test_route_weights_of_far_logits(E, k):
    """A weight's relative error does not grow with its logit's distance.

    Rows of two experts that are not barred, logits 0 and d (their difference is exact).  With the
    hardware's exponential good to 1 ulp = 2 x 2^-24, e^d is a square (2 x 2 and its rounding 1) whose
    factor holds the exponent's rounding error to first order (1, and 1 for that and all of second order):
    7 x 2^-24.  The sum 1 + e^d adds its rounding and e^-5 x 7, the quotient its rounding: 10 x 2^-24.
    The gradient of g = (0, 1) over all experts, p (1 - w): p is a term (7) times 1 / sum (2.1), rounded
    (1); 1 - w with w <= e^-5 is off by 1.1, the product by 1: 13 x 2^-24."""
    T = 4000
    rng = np.random.default_rng(E)
    d = -np.exp(rng.uniform(np.log(5), np.log(85), T)).astype(np.float32)  # (p stays a normal number)
    first = rng.integers(0, E, T)
    other = (first + 1 + rng.integers(0, E - 1, T)) % E
    for dtype in (F32, F16):
        far = torch.from_numpy(d).to(dtype)
        logits = torch.full((T, E), -float("inf"), dtype=dtype)
        logits[torch.arange(T), torch.from_numpy(first)] = 0.0
        logits[torch.arange(T), torch.from_numpy(other)] = far
        logits = logits.to(DEV)
        term = np.exp(far.double().numpy())
        w1 = term / (1 + term)
        for renormalise in (True, False):
            weights, ids = rows.route_forward(logits, k, renormalise)
            want_ids = np.full((T, k), -1, dtype=np.int32)
            want_ids[:, 0], want_ids[:, 1] = first, other
            assert np.array_equal(ids.cpu().numpy(), want_ids)
            _near(weights[:, 1], w1, 10 * U * w1, f"{dtype} renormalise={renormalise}")
            _near(weights[:, 0], 1 / (1 + term), 3 * U * np.ones(T), "the larger weight")
            if dtype == F32:
                g = torch.zeros((T, k), device=DEV)
                g[:, 1] = 1.0
                grad = rows.route_backward(g, logits, weights, ids, False)
                got = grad[torch.arange(T), torch.from_numpy(other)]
                want = w1 * (1 - w1)
                _near(got, want, 13 * U * want, f"gradient, renormalise={renormalise}")


def test_route_of_the_farthest_logits():
    """Logits whose difference overflows, and infinite ones, weigh what e^d says."""
    big, inf = 3.4e38, float("inf")
    logits = torch.tensor([[big, -big, 0.0], [-big, -big, -big], [0.0, -150.0, -103.0], [-inf, -inf, -inf],
                           [-inf, -big, -inf], [-big, inf, 0.0]], device=DEV)
    for renormalise in (True, False):
        w, ids = rows.route_forward(logits, 2, renormalise)
        assert ids.tolist() == [[0, 2], [0, 1], [0, 2], [-1, -1], [1, -1], [1, 2]]
        assert w[0].tolist() == [1.0, 0.0] and w[3].tolist() == [0.0, 0.0] and w[4].tolist() == [1.0, 0.0]
        share = 0.5 if renormalise else 1 / 3
        assert (w[1] - share).abs().max() <= 2 * U
        assert w[2, 0] == 1.0 and abs(float(w[2, 1]) - np.exp(-103.0)) <= 2.0 ** -149  # (its smallest numbers)
        assert torch.isnan(w[5]).all()
        grad = rows.route_backward(torch.ones((5, 2), device=DEV), logits[:5], w[:5], ids[:5], renormalise)
        assert torch.isfinite(grad).all() and not grad[3].any()


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(37, 8, 8), (35, 16, 12), (50, 16, 4), (33, 20, 4), (19, 32, 12), (18, 33, 9),
                                   (18, 128, 12), (18, 256, 12), (18, 256, 13), (18, 256, 3)])
def test_route_on_both_sides_of_the_list(T, E, k, dtype, renormalise):
    """Every width that 16 lanes take, both ways to the largest, several blocks with a partial last one."""
    plain.test_route(T, E, k, dtype, renormalise)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(37, 256, 8), (37, 40, 12), (70, 64, 4), (37, 32, 5)])
def test_route_rows_whose_candidates_overflow_the_list(T, E, k, dtype):
    """Rows of equal logits (more candidates than are listed, or just as many) among plain ones of a wave."""
    logits = plain._logits(T, E, dtype, 3)
    logits[1::4] = 0.5
    logits[6::8, E // 2:] = 2.0
    for renormalise in (True, False):
        w, ids = rows.route_forward(logits, k, renormalise)
        want_w, want_ids = ref.route_ref(_np(logits), k, renormalise)
        assert np.array_equal(ids.cpu().numpy(), want_ids)
        rel = np.take_along_axis(plain._route_rel(_np(logits), E), want_ids, 1)
        _near(w, want_w, rel * want_w, "weights")


# ------------------------------------------------------------------ dispatch

@pytest.mark.parametrize("E", [511, 512, 1023, 1024])
@pytest.mark.parametrize("T,k", [(341, 3), (128, 8), (205, 5), (1024, 1), (100, 7)])
def test_dispatch_on_both_sides_of_one_launch(T, k, E):
    """1023, 1024 and 1025 slots, and tables of digits from half full to one key too many."""
    say(f"dispatch T={T} k={k} E={E}")
    for C, dtype, kdt, kind in ((24, BF16, torch.int32, "even"), (5, F32, torch.int64, "even"),
                                (8, F16, torch.int32, "one"), (130, BF16, torch.int64, "low")):
        ids = _ids(T, k, E, T + E, kind) if kind != "low" else np.random.default_rng(E).integers(-3, 9, (T, k))
        ids.reshape(-1)[::17] = E  # (dropped like -1, the first key past the table)
        x = _normal(T, C, dtype=dtype, seed=1)
        got, plan = rows.dispatch_forward(x, torch.from_numpy(ids).to(kdt).to(DEV), E)
        want, wplan = ref.dispatch_ref(_np(x), ids, E)
        _same_plan(plan, wplan, kind)
        assert np.array_equal(_np(got), want), kind
        again, _ = rows.dispatch_forward(x, plan)
        assert torch.equal(again, got)


# ------------------------------------------------------------------- sorting

@pytest.mark.parametrize("n", [24, 8192, 8193, 300001])
@pytest.mark.parametrize("n_keys", [(1 << 30) + 5, (1 << 31) - 2])
def test_sort_by_keys_of_four_passes(n, n_keys):
    """The most keys there may be; their offsets (4 and 8 GiB) are compared around every key that occurs."""
    say(f"sort_keys n={n} n_keys={n_keys}")
    g = torch.Generator(device=DEV).manual_seed(n)
    keys = torch.randint(-(1 << 20), (1 << 31) + (1 << 20), (n,), generator=g, device=DEV)
    keys[:12] = torch.tensor([0, n_keys - 1, n_keys, -1, n_keys + 1, -(1 << 31), (1 << 31) - 1, 1, 1 << 32, 1 << 40,
                              (1 << 63) - 1, n_keys - 1], device=DEV)
    keys[n // 2:n // 2 + n // 8] = n_keys // 3  # a frequent one
    plan = rows.sort_keys(keys, n_keys)
    ordered, order = torch.sort(torch.where((keys >= 0) & (keys < n_keys), keys, n_keys), stable=True)
    assert torch.equal(plan.order.long(), order)
    assert torch.equal(plan.position[order].long(), torch.arange(n, device=DEV))
    assert plan.offsets.numel() == n_keys + 1
    near = torch.cat([ordered - 1, ordered, ordered + 1, torch.arange(0, n_keys, 104729, device=DEV)]).clamp(0, n_keys)
    assert torch.equal(plan.offsets[near].long(), torch.searchsorted(ordered, near))


# ------------------------------------------------------------------- streams

def test_values_on_another_stream():
    """Every call with a stream argument, by value, its inputs ready before."""
    T, k, E, V = 500, 3, 7, 90
    x, g = _normal(T, 64), _normal(T, 64, seed=1)
    ids, tids = torch.from_numpy(_ids(T, k, E, 1)).to(DEV), torch.from_numpy(plain._keys(T, V, 2)).to(DEV)
    table, logits, w = _normal(V, 64, seed=2), _normal(T, E, seed=3), _normal(T, k, seed=4)

    def calls(**on):
        r, plan = rows.dispatch_forward(x, ids, E, **on)
        again, _ = rows.dispatch_forward(x, plan, **on)
        out = rows.combine_forward(r, w, plan, **on)
        grads = rows.combine_backward(g, r, w, plan, **on)
        weights, best = rows.route_forward(logits, k, **on)
        key = rows.sort_keys(tids, V, **on)
        e = rows.embed_forward(table, tids, 2.0, **on)
        return [r, plan.order, plan.position, plan.offsets, again, out, *grads, rows.dispatch_backward(r, plan, k, **on),
                weights, best, rows.route_backward(w, logits, weights, best, **on), key.order, key.position,
                key.offsets, e, rows.embed_backward(e, tids, V, 2.0, **on)]

    want = calls()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for s in (side, side.cuda_stream):
        got = calls(stream=s)
        side.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), i
