"""Row operators on the GPU against their float64 oracle.

Tolerances: a sum of m products formed in float32 in any order is off by at
most (m + 1) 2^-24 times the sum of its terms' magnitudes (to first order;
m + 2 covers the higher ones at these lengths), and storing rounds by half a
step of the type (finfo.eps / 2 of the value, half of its smallest number near
zero).  Moves are exact.
"""

import numpy as np
import pytest
import torch

from _gpu import DEV, say
from oracle import rows_ref as ref
from paper_2211_17111_amd import bevpool as bp
from paper_2211_17111_amd import rows

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
U = 2.0 ** -24


def _np(t):
    return t.detach().double().cpu().numpy()


def _normal(*shape, dtype=F32, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).to(DEV)


def _half_step(want, dtype):
    """Half a step of the type at every value."""
    f = torch.finfo(dtype)
    return np.abs(want) * f.eps / 2 + f.smallest_normal * f.eps / 2


def _near(got, want, bound, label=""):
    assert tuple(got.shape) == want.shape, f"{label}: {tuple(got.shape)} != {want.shape}"
    err = np.abs(_np(got) - want)
    bad = ~(err <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{label}: {int(bad.sum())} of {err.size} out of tolerance, first at {i}: got "
                             f"{_np(got)[i]}, want {want[i]}, bound {np.broadcast_to(bound, err.shape)[i]}")


def _same_plan(plan, want, label=""):
    for k in ("order", "position", "offsets"):
        got = getattr(plan, k).cpu().numpy()
        assert got.dtype == np.int32
        assert np.array_equal(got, want[k]), f"{label} {k}"


def _keys(n, n_keys, seed, kind="even"):
    rng = np.random.default_rng(seed)
    if kind == "even":
        return rng.integers(-max(1, n_keys // 8), n_keys + max(1, n_keys // 8), n)
    if kind == "one":
        return np.full(n, n_keys - 1)
    if kind == "none":
        return np.full(n, -1)
    if kind == "falling":
        return np.arange(n)[::-1] % n_keys
    return np.minimum((n_keys + 1.0) ** rng.random(n) - 1, n_keys - 1).astype(np.int64)  # "zipf"


# ------------------------------------------------------------------- sorting

@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 255, 257, 1000, 2047, 2048, 2049, 4096, 4097, 8191, 8192, 8193,
                               70001])
@pytest.mark.parametrize("n_keys", [1, 2, 7, 255, 256, 1023, 1024, 5000, (1 << 20) + 3])
def test_sort_keys(n, n_keys):
    say(f"sort_keys n={n} n_keys={n_keys}")
    for kind, dtype in (("even", torch.int32), ("even", torch.int64), ("zipf", torch.int32)):
        keys = _keys(n, n_keys, n + n_keys, kind)
        plan = rows.sort_keys(torch.from_numpy(keys).to(dtype).to(DEV), n_keys)
        _same_plan(plan, ref.sort_keys_ref(keys, n_keys), f"{kind} {dtype}")


@pytest.mark.parametrize("kind", ["one", "none", "falling"])
@pytest.mark.parametrize("n,n_keys", [(5, 3), (3000, 64), (3000, 1 << 18), (40000, 300)])
def test_sort_keys_shapes(kind, n, n_keys):
    keys = _keys(n, n_keys, 0, kind)
    plan = rows.sort_keys(torch.from_numpy(keys).to(torch.int32).to(DEV), n_keys)
    _same_plan(plan, ref.sort_keys_ref(keys, n_keys), kind)


def test_sort_keys_extreme_values():
    """Keys far outside are dropped whatever their low bits say."""
    for n_keys in (5, 3000, 1 << 22, (1 << 31) - 2):
        if n_keys > 1 << 23:
            continue  # (offsets of 2^31 keys are 8 GiB)
        base = [0, n_keys - 1, n_keys, -1, n_keys + 1, -(1 << 31), (1 << 31) - 1, 1]
        wide = base + [1 << 32, (1 << 32) + 1, -(1 << 32), (1 << 63) - 1, -(1 << 63), (1 << 40) + 3]
        for vals, dtype in ((base, torch.int32), (wide, torch.int64)):
            keys = np.array(vals * 3, dtype=np.int64)
            plan = rows.sort_keys(torch.from_numpy(keys).to(dtype).to(DEV), n_keys)
            _same_plan(plan, ref.sort_keys_ref(keys, n_keys), f"{n_keys} {dtype}")


@pytest.mark.parametrize("n", [262144, 262145, 1500007])
@pytest.mark.parametrize("n_keys", [3, 900, 70000, 1 << 21])
def test_sort_many_keys(n, n_keys):
    """More groups of tiles than a block adds up itself, against torch's stable sort."""
    say(f"sort_keys n={n} n_keys={n_keys}")
    g = torch.Generator(device=DEV).manual_seed(n + n_keys)
    keys = torch.randint(-n_keys // 9 - 1, n_keys + n_keys // 9 + 1, (n,), generator=g, device=DEV)
    keys[n // 3:n // 2] = n_keys // 2  # a frequent one
    plan = rows.sort_keys(keys, n_keys)
    k = torch.where((keys >= 0) & (keys < n_keys), keys, n_keys)
    ordered, order = torch.sort(k, stable=True)
    assert torch.equal(plan.order.long(), order)
    assert torch.equal(plan.position[order].long(), torch.arange(n, device=DEV))
    assert torch.equal(plan.offsets.long(), torch.searchsorted(ordered, torch.arange(n_keys + 1, device=DEV)))


# -------------------------------------------------------------------- router

def _logits(T, E, dtype, seed, kind="plain"):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn((T, E), generator=g) * 3
    if kind == "ties":
        l = torch.randint(-2, 3, (T, E), generator=g).float() * 0.5
        l[l == 0] = torch.where(torch.rand(int((l == 0).sum()), generator=g) < 0.5, 0.0, -0.0)
    if kind == "masked":
        l[torch.rand((T, E), generator=g) < 0.5] = -float("inf")
        l[0] = -float("inf")
        l[-1, 1:] = -float("inf")
    if kind == "lowest":
        l[torch.rand((T, E), generator=g) < 0.5] = torch.finfo(dtype).min
        l[0] = torch.finfo(dtype).min
    return l.to(dtype).to(DEV)


def _route_rel(l, E):
    """Relative error of a weight exp(l - m) / sum: two roundings of the exponent
    (each |l - m| 2^-24 of the term), exp's 2 ulp, the sum's (E + 1) 2^-24 and its
    terms' own errors, the quotient; l - m is taken for the row."""
    top = np.max(np.where(np.isfinite(l), l, -np.inf), axis=1, keepdims=True)
    d = np.minimum(np.where(np.isfinite(top), top, 0) - l, 104)  # (terms below e^-104 are 0 in float32)
    return U * (4 * np.where(np.isfinite(d), d, 0) + 2 * E + 16)


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 2, 2), (1, 64, 6), (7, 5, 3), (33, 16, 2), (9, 60, 4), (5, 64, 64),
                                   (10, 65, 8), (6, 128, 8), (4, 200, 64), (5, 256, 8), (3, 257, 12), (2, 512, 10),
                                   (3, 1000, 33), (2, 1024, 64)])
def test_route(T, E, k, dtype, renormalise):
    say(f"route T={T} E={E} k={k} {dtype} renormalise={renormalise}")
    for kind in ("plain", "ties", "masked", "lowest"):
        logits = _logits(T, E, dtype, T * E + k, kind)
        l = _np(logits)
        want_w, want_ids = ref.route_ref(l, k, renormalise)
        weights, ids = rows.route_forward(logits, k, renormalise)
        assert weights.dtype == F32 and ids.dtype == torch.int32
        assert np.array_equal(ids.cpu().numpy(), want_ids), kind
        rel = _route_rel(l, E)
        chosen = np.where(want_ids >= 0, want_ids, 0)
        w_rel = np.take_along_axis(rel, chosen, 1)
        _near(weights, want_w, w_rel * want_w + 1e-44, kind)
        # the gradient, at the kernel's own weights
        g = _normal(T, k, seed=5)
        grad = rows.route_backward(g, logits, weights, ids, renormalise)
        assert grad.dtype == dtype
        want = ref.route_backward_ref(_np(g), l, k, renormalise)
        gj = np.where(want_ids >= 0, _np(g), 0)
        s_mag = (np.abs(gj) * want_w).sum(1, keepdims=True)
        s_err = (np.abs(gj) * want_w * (w_rel + (k + 2) * U)).sum(1, keepdims=True)
        G = np.zeros((T, E))
        over = np.zeros((T, E))
        for t in range(T):
            for j, e in enumerate(want_ids[t]):
                if e >= 0:
                    G[t, e] = abs(gj[t, j])
                    over[t, e] = 1
        with np.errstate(invalid="ignore"):
            top = np.max(np.where(np.isfinite(l), l, -np.inf), axis=1, keepdims=True)
            p = np.where(np.isfinite(l), np.exp(np.minimum(l - np.where(np.isfinite(top), top, 0), 0)), 0)
        p = p * over if renormalise else p
        p = p / np.maximum(p.sum(1, keepdims=True), 1e-300)
        bound = p * ((rel + 4 * U) * (G + s_mag) + s_err) + _half_step(want, dtype) + 1e-44
        _near(grad, want, bound, f"{kind} gradient")


def test_route_nan_and_inf():
    nan, inf = float("nan"), float("inf")
    logits = torch.tensor([[1., nan, 3., 2.], [inf, 0., 1., 2.], [nan] * 4, [1., 2., 3., 4.], [-inf, nan, -inf, -inf]],
                          device=DEV)
    for renormalise in (True, False):
        w, ids = rows.route_forward(logits, 2, renormalise)
        assert ids.tolist() == [[2, 3], [0, 3], [-1, -1], [3, 2], [-1, -1]]
        assert torch.isnan(w[[0, 2, 4]]).all() and torch.isnan(w[1, 0])
        assert torch.isfinite(w[3]).all()
        g = rows.route_backward(torch.ones_like(w), logits, w, ids, renormalise)
        assert torch.isnan(g[0, 2]) and torch.isfinite(g[3]).all()


def test_route_strided_rows():
    wide = _logits(9, 100, BF16, 3)
    w, ids = rows.route_forward(wide[:, 7:47], 4)
    w2, ids2 = rows.route_forward(wide[:, 7:47].contiguous(), 4)
    assert torch.equal(w, w2) and torch.equal(ids, ids2)
    one = wide[:1, :40].expand(5, 40)
    w, ids = rows.route_forward(one, 3, False)
    assert torch.equal(w, w[:1].expand(5, 3)) and torch.equal(ids, ids[:1].expand(5, 3))
    g = rows.route_backward(torch.ones_like(w), one, w, ids, False)
    assert torch.equal(g, g[:1].expand(5, 40))


# ------------------------------------------------------- dispatch and combine

def _ids(T, k, E, seed, kind="even"):
    rng = np.random.default_rng(seed)
    if kind == "none":
        return np.full((T, k), -1)
    if kind == "one":
        return np.full((T, k), E - 1)
    return rng.integers(-1, E, (T, k))


SHAPES = [(0, 2, 4, 16), (1, 1, 1, 1), (1, 6, 64, 2048), (3, 2, 5, 7), (5, 8, 16, 8), (17, 3, 9, 33), (64, 4, 8, 80),
          (130, 2, 300, 1001), (300, 8, 128, 64), (33, 5, 2000, 130), (700, 12, 40, 24), (40, 9, 12, 4100)]


@pytest.mark.parametrize("kind", ["even", "one", "none"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,C", SHAPES)
def test_dispatch_and_combine(T, k, E, C, dtype, kind):
    say(f"dispatch/combine T={T} k={k} E={E} C={C} {dtype} {kind}")
    ids = _ids(T, k, E, T + k, kind)
    kdt = torch.int64 if T % 2 else torch.int32
    x = _normal(T, C, dtype=dtype, seed=1)
    got, plan = rows.dispatch_forward(x, torch.from_numpy(ids).to(kdt).to(DEV), E)
    want, wplan = ref.dispatch_ref(_np(x), ids, E)
    _same_plan(plan, wplan)
    assert got.dtype == dtype and np.array_equal(_np(got), want)
    again, same = rows.dispatch_forward(x, plan)
    assert same is plan and torch.equal(again, got)

    g = _normal(T * k, C, dtype=dtype, seed=2)
    ones = np.ones((T, k))
    want, mag = ref.combine_ref(_np(g), ones, wplan)
    _near(rows.dispatch_backward(g, plan, k), want, (k + 2) * U * mag + _half_step(want, dtype), "dispatch gradient")

    # combine: weights in float32 and in the rows' type, results in it and in float32
    y, go = _normal(T * k, C, dtype=dtype, seed=3), _normal(T, C, seed=4)
    for wdt in {F32, dtype}:
        w = _normal(T, k, dtype=wdt, seed=5)
        want, mag = ref.combine_ref(_np(y), _np(w), wplan)
        for odt in {F32, dtype}:
            out = rows.combine_forward(y, w, plan, odt)
            assert out.dtype == odt
            _near(out, want, (k + 2) * U * mag + _half_step(want, odt), f"combine {wdt} {odt}")
            gout = go.to(odt)
            grad_rows, grad_w = rows.combine_backward(gout, y, w, plan)
            wr, ww, wmag = ref.combine_backward_ref(_np(gout), _np(y), _np(w), wplan)
            assert grad_rows.dtype == dtype and grad_w.dtype == wdt
            _near(grad_rows, wr, U * np.abs(wr) + _half_step(wr, dtype) * (1 + 2 * U), "gradient of the rows")
            _near(grad_w, ww, (C + 2) * U * wmag + _half_step(ww, wdt) * (1 + 2 * U), "gradient of the weights")
            only, none = rows.combine_backward(gout, y, w, plan, need_weights=False)
            assert none is None and torch.equal(only, grad_rows)
            none, only = rows.combine_backward(gout, y, w, plan, need_rows=False)
            assert none is None and torch.equal(only, grad_w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,C", [(5003, 4, 1027), (2100, 9, 1024), (40000, 3, 300)])
def test_many_rows(T, k, C, dtype):
    """Sizes past the caches, where rows are streamed: against float64 on the device."""
    say(f"many rows T={T} k={k} C={C} {dtype}")
    E = 40
    ids = torch.from_numpy(_ids(T, k, E, 8)).to(DEV)
    x, y = _normal(T, C, dtype=dtype), _normal(T * k, C, dtype=dtype, seed=1)
    assert y.numel() * y.element_size() > 32 << 20
    w, g = _normal(T, k, seed=2), _normal(T, C, dtype=dtype, seed=3)
    r, plan = rows.dispatch_forward(x, ids, E)
    kept = int(plan.offsets[-1])
    assert torch.equal(r[:kept], x[plan.order[:kept].long() // k]) and not r[kept:].any()
    pos = plan.position.long().view(T, k)
    on = (pos < kept)[..., None]
    mine = torch.where(on, y[pos], 0).double()

    def check(got, want, bound, label):
        half = want.abs() * torch.finfo(got.dtype).eps / 2 + torch.finfo(got.dtype).smallest_normal
        assert ((got.double() - want).abs() <= bound + half * (1 + 2 * U)).all(), label

    terms = w.double()[..., None] * mine
    check(rows.combine_forward(y, w, plan), terms.sum(1), (k + 2) * U * terms.abs().sum(1), "combine")
    check(rows.dispatch_backward(y, plan, k), mine.sum(1), (k + 2) * U * mine.abs().sum(1), "dispatch gradient")
    grad_rows, grad_w = rows.combine_backward(g, y, w, plan)
    want = torch.where(on, w.double()[..., None] * g.double()[:, None], 0.0)
    check(grad_rows[pos.view(-1)].view(T, k, C), want, U * want.abs(), "gradient of the rows")
    terms = mine * g.double()[:, None]
    check(grad_w, terms.sum(2), (C + 2) * U * terms.abs().sum(2), "gradient of the weights")
    V = 1000
    eids = torch.randint(-1, V, (T * k,), device=DEV)
    want, mag = torch.zeros(V + 1, C, dtype=torch.float64, device=DEV), torch.zeros(V + 1, C, dtype=torch.float64, device=DEV)
    row = torch.where(eids >= 0, eids, V)
    want.index_add_(0, row, y.double())
    mag.index_add_(0, row, y.double().abs())
    n = torch.bincount(row, minlength=V + 1)[:V, None]
    check(rows.embed_backward(y, eids, V), want[:V], (n + 2) * U * mag[:V], "embedding gradient")


def test_rows_behind_the_kept_ones_are_not_used():
    """Infinities and NaN in rows of dropped slots reach nothing."""
    T, k, E, C = 20, 3, 4, 40
    ids = torch.from_numpy(_ids(T, k, E, 3)).to(DEV)
    _, plan = rows.dispatch_forward(_normal(T, C), ids, E)
    kept = int(plan.offsets[-1])
    assert kept < T * k
    y, w, g = _normal(T * k, C, seed=1), _normal(T, k, seed=2), _normal(T, C, seed=3)
    clean = rows.combine_forward(y, w, plan), *rows.combine_backward(g, y, w, plan), rows.dispatch_backward(y, plan, k)
    y[kept:] = float("nan")
    y[-1] = float("inf")
    w.view(-1)[plan.order[kept:].long()] = float("nan")
    dirty = rows.combine_forward(y, w, plan), *rows.combine_backward(g, y, w, plan), rows.dispatch_backward(y, plan, k)
    for a, b in zip(clean, dirty):
        assert torch.equal(a, b)


def test_nan_and_inf_are_moved_as_they_are():
    bits = torch.tensor([0x7fc1, 0xffc3, 0x7f80, 0x8000, 1], dtype=torch.int32).to(torch.int16).to(DEV)
    x = bits.view(BF16).repeat(2, 3)
    got, plan = rows.dispatch_forward(x, torch.tensor([[1, 0], [0, 2]], device=DEV), 3)
    assert torch.equal(got.view(torch.int16), x.view(torch.int16)[plan.order.long() // 2])


def test_strided_and_expanded_rows():
    T, k, E, C = 37, 3, 6, 45
    ids = torch.from_numpy(_ids(T, k, E, 5)).to(DEV)
    for dtype in TYPES:
        wide = _normal(T, 2 * C + 3, dtype=dtype)
        x = wide[:, 5:5 + C]
        a, plan = rows.dispatch_forward(x, ids, E)
        b, _ = rows.dispatch_forward(x.contiguous(), ids, E)
        assert torch.equal(a, b)
        one, _ = rows.dispatch_forward(x[:1].expand(T, C), plan)
        kept = int(plan.offsets[-1])
        assert torch.equal(one[:kept], x[:1].expand(kept, C)) and not one[kept:].any()
        wide = _normal(T * k, C + 11, dtype=dtype, seed=1)
        y, w = wide[:, 3:3 + C], _normal(T, k, seed=2)
        assert torch.equal(rows.combine_forward(y, w, plan), rows.combine_forward(y.contiguous(), w, plan))
        assert torch.equal(rows.dispatch_backward(y, plan, k), rows.dispatch_backward(y.contiguous(), plan, k))
        g = wide[:T, 1:1 + C]
        for p, q in zip(rows.combine_backward(g, y, w, plan),
                        rows.combine_backward(g.contiguous(), y.contiguous(), w, plan)):
            assert torch.equal(p, q)


# ----------------------------------------------------------------- embedding

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["even", "one", "none", "zipf"])
@pytest.mark.parametrize("n,V,C", [(0, 3, 8), (1, 1, 1), (1, 1000, 64), (5, 7, 3), (64, 16, 80), (300, 40, 33),
                                   (2000, 3, 130), (5000, 2, 16), (1000, 3000, 24), (700, 1100, 1001), (9000, 50, 40),
                                   (30, 20, 4100)])
def test_embed(n, V, C, dtype, kind):
    say(f"embed n={n} V={V} C={C} {dtype} {kind}")
    ids = _keys(n, V, n + V, kind)
    kdt = torch.int32 if n % 2 else torch.int64
    dids = torch.from_numpy(ids).to(kdt).to(DEV)
    table = _normal(V, C, dtype=dtype, seed=1)
    scale = 1.0 if n % 3 == 0 else 3.7
    want = ref.embed_ref(_np(table), ids, float(np.float32(scale)))
    for odt in {F32, dtype}:
        out = rows.embed_forward(table, dids, scale, odt)
        assert out.dtype == odt
        _near(out, want, U * np.abs(want) + _half_step(want, odt) * (1 + 2 * U), f"embed {odt}")
        g = _normal(n, C, dtype=odt, seed=2)
        for gdt in {dtype, odt, F32}:
            grad = rows.embed_backward(g, dids, V, scale, gdt)
            wg, mag, count = ref.embed_backward_ref(_np(g), ids, V, float(np.float32(scale)))
            assert grad.dtype == gdt
            _near(grad, wg, (count[:, None] + 2) * U * mag + _half_step(wg, gdt) * (1 + 4 * U), f"gradient {odt} {gdt}")
            assert not grad[torch.from_numpy(count == 0).to(DEV)].any()


def test_embed_shapes_and_strides():
    table = _normal(30, 50)[:, 4:29]
    ids = torch.randint(-1, 31, (2, 3, 4), device=DEV)
    out = rows.embed_forward(table, ids, 2.0)
    assert out.shape == (2, 3, 4, 25)
    assert torch.equal(out, rows.embed_forward(table.contiguous(), ids.view(-1), 2.0).view(2, 3, 4, 25))
    g = _normal(24, 60, seed=1)[:, 10:35]
    a = rows.embed_backward(g, ids.view(-1), 30, 2.0)
    assert torch.equal(a, rows.embed_backward(g.contiguous().view(2, 3, 4, 25), ids, 30, 2.0))
    one = rows.embed_forward(table, torch.tensor(3, device=DEV))
    assert one.shape == (25,) and torch.equal(one, table[3])
    assert torch.equal(rows.embed_backward(one, torch.tensor(3, device=DEV), 30)[3], one)
    row = _normal(1, 25, seed=2)
    e = rows.embed_backward(row.expand(24, 25), ids.view(-1), 30)
    assert torch.equal(e, rows.embed_backward(row.expand(24, 25).contiguous(), ids.view(-1), 30))


def test_embed_places_past_32_bits():
    """Rows that lie more than 2^32 bytes and elements into their matrices."""
    V, C = (1 << 20) + 9, 4104  # 4.3e9 elements, 8.6 GB
    table = torch.empty((V, C), dtype=BF16, device=DEV)
    ids = torch.tensor([V - 1, 0, V // 2, V - 1, V], device=DEV)
    table[ids[:3]] = _normal(3, C, dtype=BF16)
    out = rows.embed_forward(table, ids)
    assert torch.equal(out[:4], table[ids[:4]]) and not out[4].any()
    del table
    grad = rows.embed_backward(out, ids, V)
    assert torch.equal(grad[V - 1], (out[0].float() + out[3].float()).to(BF16))
    assert torch.equal(grad[V // 2], out[2]) and torch.equal(grad[0], out[1])
    assert not grad[1:V // 2].any() and not grad[V // 2 + 1:V - 1].any()


@pytest.mark.parametrize("n,V,C,kind", [(400000, 5, 12, "zipf"), (400000, 300000, 20, "even"), (300000, 2000, 40, "one")])
def test_embed_gradient_of_many_slots(n, V, C, kind):
    """Long ranges, and ids of hundreds of ranges, against float64 on the device."""
    say(f"embedding gradient n={n} V={V} C={C} {kind}")
    ids = torch.from_numpy(_keys(n, V, 3, kind)).to(DEV)
    g = _normal(n, C, seed=1)
    row = torch.where((ids >= 0) & (ids < V), ids, V)
    want, mag = (torch.zeros(V + 1, C, dtype=torch.float64, device=DEV) for _ in range(2))
    want.index_add_(0, row, g.double())
    mag.index_add_(0, row, g.double().abs())
    count = torch.bincount(row, minlength=V + 1)[:V, None]
    got = rows.embed_backward(g, ids, V)
    assert ((got.double() - want[:V]).abs() <= (count + 2) * U * mag[:V] + 1e-30).all()
    assert not got[count[:, 0] == 0].any()


def test_dispatch_and_combine_past_32_bits():
    """Slots' rows that lie more than 2^32 elements in."""
    T, k, C, E = (1 << 18) + 5, 4, 4104, 8  # 4.3e9 elements of rows
    x = torch.randn((T, C), dtype=BF16, device=DEV)
    ids = torch.randint(0, E, (T, k), device=DEV)
    r, plan = rows.dispatch_forward(x, ids, E)
    for q in (0, T * k // 2, T * k - 2, T * k - 1):
        assert torch.equal(r[q], x[int(plan.order[q]) // k]), q
    w = torch.full((T, k), 0.25, device=DEV)
    assert torch.equal(rows.combine_forward(r, w, plan), x)  # (four quarters: exact)
    grad_rows, grad_w = rows.combine_backward(x, r, w, plan)
    for q in (0, T * k // 2, T * k - 1):
        assert torch.equal(grad_rows[q], (0.25 * x[int(plan.order[q]) // k].float()).to(BF16)), q
    t = torch.tensor([0, T // 2, T - 1], device=DEV)
    want = x[t].double().square().sum(1, keepdim=True)
    assert ((grad_w[t].double() - want).abs() <= (C + 2) * U * want).all()
    del grad_rows, grad_w
    back = rows.dispatch_backward(r, plan, k)
    assert torch.equal(back, (4 * x.float()).to(BF16))


# ------------------------------------------------------------ used together

def _layer(x, logits, w1, k, E, renormalise=True):
    """A layer of experts, each one matrix."""
    weights, ids = rows.route(logits, k, renormalise)
    r, plan = rows.dispatch(x, ids, E)
    cut = plan.offsets.tolist()
    y = torch.cat([r[cut[e]:cut[e + 1]] @ w1[e] for e in range(E)] + [r[cut[E]:]])
    return rows.combine(y, weights, plan)


def test_expert_layer_on_embedded_tokens():
    """embed -> route -> dispatch -> experts -> combine, against the same written
    with dense masks in float64, values and all gradients."""
    T, V, C, E, k = 50, 40, 24, 6, 2
    ids = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(0)).to(DEV)
    ids[::9] = -1
    leaves = [_normal(V, C, seed=1), _normal(C, E, seed=2), _normal(E, C, C, seed=3)]
    target = _normal(T, C, seed=4)
    table, wr, w1 = (t.clone().requires_grad_() for t in leaves)
    x = rows.embed(table, ids, 2.0)
    out = _layer(x, x @ wr, w1, k, E)
    (out * target).sum().backward()

    t64, r64, m64 = (t.double().cpu().requires_grad_() for t in leaves)
    i = ids.cpu()
    x64 = torch.where((i >= 0)[:, None], t64[i.clamp_min(0)] * 2.0, 0.0)
    l64 = x64 @ r64
    # (rows of padding have equal logits: the lower experts are chosen)
    top = torch.sort(l64, dim=1, descending=True, stable=True).indices[:, :k]
    mask = torch.zeros_like(l64).scatter_(1, top, 1.0)
    p = torch.exp(l64 - l64.amax(1, keepdim=True)) * mask
    p = p / p.sum(1, keepdim=True)
    out64 = torch.einsum("te,td,edc->tc", p, x64, m64)
    (out64 * target.double().cpu()).sum().backward()
    # A logit is a sum of C = 24 products of magnitude 60 in all at most, so it is off by at most
    # 26 x 60 x 2^-24, and a weight by that relative to itself; the experts' products and the sums of
    # their gradients add (C + 2) 2^-24 each: 2000 x 2^-24 of the tensor's largest value covers them.
    for a, b in ((out, out64), (table.grad, t64.grad), (wr.grad, r64.grad), (w1.grad, m64.grad)):
        err = (a.detach().double().cpu() - b.detach()).abs().max()
        assert err <= 2000 * U * b.detach().abs().max(), float(err / b.detach().abs().max())


def test_gradients_against_differences():
    """Central differences of the float64 oracle along random directions."""
    T, E, k, C, V = 12, 10, 3, 17, 9
    rng = np.random.default_rng(0)
    for renormalise in (True, False):
        l = rng.permuted(np.linspace(-2, 2, E)[None].repeat(T, 0), axis=1)  # gaps of 0.44: no choice changes
        c, d, h = rng.normal(size=(T, k)), rng.normal(size=(T, E)), 1e-4
        diff = sum(s * (ref.route_ref(l + s * h * d, k, renormalise)[0] * c).sum() for s in (1, -1)) / (2 * h)
        logits = torch.from_numpy(l).float().to(DEV).requires_grad_()
        w, _ = rows.route(logits, k, renormalise)
        (w * torch.from_numpy(c).float().to(DEV)).sum().backward()
        got = (_np(logits.grad) * d).sum()
        assert abs(got - diff) <= 1e-5 * np.abs(_np(logits.grad) * d).sum() + 1e-7
    ids = _ids(T, k, E, 1)
    dids = torch.from_numpy(ids).to(DEV)
    x, y, w, g = (_normal(*s, seed=i).requires_grad_() for i, s in enumerate([(T, C), (T * k, C), (T, k), (T, C)]))
    r, plan = rows.dispatch(x, dids, E)
    (r * y.detach()).sum().backward()
    wplan = ref.sort_keys_ref(ids, E)
    # the maps are linear in each argument: f(x + d) - f(x) is the derivative along d
    d = _np(_normal(T, C, seed=9))
    assert np.isclose((ref.dispatch_ref(d, ids, E)[0] * _np(y)).sum(), (_np(x.grad) * d).sum(), rtol=1e-4, atol=1e-4)
    out = rows.combine(y, w, plan)
    (out * g.detach()).sum().backward()
    dy, dw = _np(_normal(T * k, C, seed=10)), _np(_normal(T, k, seed=11))
    assert np.isclose((ref.combine_ref(dy, _np(w), wplan)[0] * _np(g)).sum(), (_np(y.grad) * dy).sum(), rtol=1e-4, atol=1e-4)
    assert np.isclose((ref.combine_ref(_np(y), dw, wplan)[0] * _np(g)).sum(), (_np(w.grad) * dw).sum(), rtol=1e-4, atol=1e-4)
    table = _normal(V, C, seed=12).requires_grad_()
    eids = torch.randint(-1, V, (40,), device=DEV)
    c = _normal(40, C, seed=13)
    (rows.embed(table, eids, 1.5) * c).sum().backward()
    dt = _np(_normal(V, C, seed=14))
    assert np.isclose((ref.embed_ref(dt, eids.cpu().numpy(), 1.5) * _np(c)).sum(), (_np(table.grad) * dt).sum(),
                      rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("dtype", TYPES)
def test_autograd_types_and_broadcast_gradients(dtype):
    """Gradients come in their leaves' types, also from an expanded gradient and a float32 result."""
    T, k, E, C = 9, 2, 4, 24
    ids = torch.from_numpy(_ids(T, k, E, 2)).to(DEV)
    x = _normal(T, C, dtype=dtype).requires_grad_()
    r, plan = rows.dispatch(x, ids, E)
    r.sum().backward()
    kept = (ids >= 0).sum(1).to(dtype)
    assert x.grad.dtype == dtype and torch.equal(x.grad, kept[:, None].expand(T, C))
    x.grad = None
    r2, same = rows.dispatch(x, plan)
    assert same is plan and torch.equal(r2, r)
    r2.sum().backward()
    assert torch.equal(x.grad, kept[:, None].expand(T, C))
    y, w = _normal(T * k, C, dtype=dtype).requires_grad_(), _normal(T, k, seed=1).requires_grad_()
    out = rows.combine(y, w, plan, F32)
    assert out.dtype == F32
    out.sum().backward()
    assert y.grad.dtype == dtype and w.grad.dtype == F32
    table = _normal(6, C, dtype=dtype).requires_grad_()
    rows.embed(table, ids.view(-1), 0.5, F32).sum().backward()
    count = torch.bincount(ids[ids >= 0], minlength=6).to(dtype) * 0.5
    assert table.grad.dtype == dtype and torch.equal(table.grad, count[:, None].expand(6, C))
    out = rows.combine(y, w.detach(), plan)
    g, = torch.autograd.grad(out.sum(), y)
    assert g.shape == y.shape
    # two uses of one leaf add up
    table.grad = None
    (rows.embed(table, ids.view(-1)).sum() + rows.embed(table, ids.view(-1)).sum()).backward()
    assert torch.equal(table.grad, 4 * count[:, None].expand(6, C))


def test_results_repeat_bit_for_bit():
    ids = torch.from_numpy(_keys(20000, 30, 1, "zipf")).to(DEV)
    g = _normal(20000, 96, dtype=BF16)
    first = rows.embed_backward(g, ids, 30, grad_dtype=F32)
    for _ in range(3):
        assert torch.equal(rows.embed_backward(g, ids, 30, grad_dtype=F32), first)


def _whole_pass(x, logits, table, tids, g, E, k):
    weights, ids = rows.route_forward(logits, k, False)
    r, plan = rows.dispatch_forward(x, ids, E)
    out = rows.combine_forward(r, weights, plan)
    grad_rows, grad_w = rows.combine_backward(g, r, weights, plan)
    grad_x = rows.dispatch_backward(grad_rows, plan, k)
    grad_l = rows.route_backward(grad_w, logits, weights, ids, False)
    e = rows.embed_forward(table, tids, 2.0)
    grad_t = rows.embed_backward(e, tids, table.shape[0], 2.0)
    return [weights, ids, r, plan.order, plan.position, plan.offsets, out, grad_rows, grad_w, grad_x, grad_l, e, grad_t]


@pytest.mark.parametrize("T,E,k,C,V", [(3, 8, 2, 64, 5), (2500, 20, 4, 72, 5000)])
def test_graph_replays_match_eager(T, E, k, C, V):
    """Every operator in one captured graph, replayed on changed inputs."""
    say(f"graph T={T}")

    def inputs(seed):
        return (_normal(T, C, dtype=BF16, seed=seed), _normal(T, E, seed=seed + 1), _normal(V, C, dtype=BF16, seed=seed + 2),
                torch.from_numpy(_keys(T, V, seed, "zipf")).to(DEV), _normal(T, C, dtype=BF16, seed=seed + 3))

    held = inputs(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _whole_pass(*held, E, k)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _whole_pass(*held, E, k)
    for seed in (10, 20, 30):
        new = inputs(seed)
        want = [t.clone() for t in _whole_pass(*new, E, k)]
        for a, b in zip(held, new):
            a.copy_(b)
        torch.cuda.synchronize()
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), f"output {i}, inputs {seed}"


def test_two_streams_at_once():
    """Two whole passes on two streams, each with its own workspaces, interleaved."""
    E, k = 16, 4
    sets = [(_normal(3000, 40, seed=s), _normal(3000, E, seed=s + 1), _normal(70, 40, seed=s + 2),
             torch.from_numpy(_keys(3000, 70, s, "zipf")).to(DEV), _normal(3000, 40, seed=s + 3)) for s in (1, 2)]
    want = [_whole_pass(*s, E, k) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(_whole_pass(*sets[i], E, k))
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            for a, b in zip(run, want[i]):
                assert torch.equal(a, b)


def test_stream_argument():
    """The stream argument: as a torch stream and as a raw handle."""
    x, ids = _normal(500, 64), torch.from_numpy(_ids(500, 3, 7, 1)).to(DEV)
    table, tids = _normal(90, 64), torch.from_numpy(_keys(500, 90, 2)).to(DEV)
    want, wplan = rows.dispatch_forward(x, ids, 7)
    wgrad = rows.embed_backward(x, tids, 90)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for s in (st, st.cuda_stream):
        got, plan = rows.dispatch_forward(x, ids, 7, stream=s)
        grad = rows.embed_backward(x, tids, 90, stream=s)
        back = rows.dispatch_backward(got, plan, 3, stream=s)
        out = rows.combine_forward(got, torch.ones(500, 3, device=DEV), plan, stream=s)
        e = rows.embed_forward(table, tids, stream=s)
        w, i = rows.route_forward(x, 2, stream=s)
        gl = rows.route_backward(w, x, w, i, stream=s)
        key = rows.sort_keys(tids, 90, stream=s)
        st.synchronize()
        assert torch.equal(got, want) and torch.equal(plan.order, wplan.order) and torch.equal(grad, wgrad)
        assert torch.equal(back, rows.dispatch_backward(want, wplan, 3))
        assert out.shape == x.shape and torch.equal(e, rows.embed_forward(table, tids))
        assert torch.equal(gl, rows.route_backward(w, x, w, i)) and torch.equal(key.order, rows.sort_keys(tids, 90).order)


def test_refusals():
    x, ids = _normal(8, 16), torch.zeros(8, 2, dtype=torch.int32, device=DEV)
    _, plan = rows.dispatch_forward(x, ids, 3)
    y, w = _normal(16, 16), _normal(8, 2)
    bad = [
        lambda: rows.sort_keys(ids.float(), 3),
        lambda: rows.sort_keys(ids.t(), 3),
        lambda: rows.route_forward(x.double(), 2),
        lambda: rows.route_forward(x.t(), 2),
        lambda: rows.route_forward(x[0], 2),
        lambda: rows.route_backward(w, x, w, ids.long()),
        lambda: rows.route_backward(w[:4], x, w, ids),
        lambda: rows.dispatch_forward(x, ids),
        lambda: rows.dispatch_forward(x, ids[:5], 3),
        lambda: rows.dispatch_forward(x, ids.view(-1), 3),
        lambda: rows.dispatch_forward(x.t(), ids, 3),
        lambda: rows.dispatch_forward(x[:5], plan),
        lambda: rows.dispatch_forward(x, ids.cpu(), 3),
        lambda: rows.dispatch_backward(y, plan, 3),
        lambda: rows.dispatch_backward(y[:8], plan, 2),
        lambda: rows.combine_forward(y, w.t(), plan),
        lambda: rows.combine_forward(y, w[:4], plan),
        lambda: rows.combine_forward(y, w.half(), plan),
        lambda: rows.combine_forward(y, w, plan, F16),
        lambda: rows.combine_forward(y[:8], w[:4], plan),
        lambda: rows.combine_forward(y, w.view(4, 4), plan),  # as many slots, otherwise grouped
        lambda: rows.dispatch_backward(y, plan, 4),
        lambda: rows.dispatch_forward(x[:4], plan),
        lambda: rows.combine_backward(x[:4], y, w.view(4, 4), plan),
        lambda: rows.combine_backward(x[:, :8], y, w, plan),
        lambda: rows.combine_backward(x.half(), y, w, plan),
        lambda: rows.combine_backward(x, y, w.cpu(), plan),
        lambda: rows.embed_forward(x, ids.t()),
        lambda: rows.embed_forward(x.half(), ids, 1.0, BF16),
        lambda: rows.embed_backward(x, ids.view(-1), 4),
        lambda: rows.embed_backward(x.half(), ids[:, 0].contiguous(), 4, 1.0, BF16),
        lambda: rows.embed_backward(_normal(8, 2, 32)[:, :, :16], ids, 4),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            raise AssertionError(f"call {i} was accepted")
    for f in (lambda: rows.sort_keys(ids, 0), lambda: rows.route_forward(x, 17), lambda: rows.route_forward(x, 0),
              lambda: rows.embed_forward(x[:0], ids)):
        with pytest.raises((bp.BevpoolError, RuntimeError)):
            f()
