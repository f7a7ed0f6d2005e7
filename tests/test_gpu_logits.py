"""Logits operators on the GPU against their float64 oracle.

Tolerances, in units of U = 2^-24 (a rounding to float32 is off by at most U
relative to its result).  A term e^-d, d = scale (m - x), is off by 2.5 d U for its
exponent (the difference, the factor scale log2 e and their product are rounded,
the factor's rounding is half as large) and 2 U for the exponential.  Partial sums
are joined in chains of at most CHAIN(V) additions, each of which may also move a
partial sum to a larger maximum (a product, an exponential): 4 U an addition.  A
logarithm is off by 2 U of itself.  Storing rounds by half a step of the type.
Terms below 2^-126 are 0.
"""

import numpy as np
import pytest
import torch

from _gpu import DEV, say
from oracle import logits_ref as ref
from paper_2211_17111_amd import logits as lg
from paper_2211_17111_amd import rows

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
U = 2.0 ** -24
TINY = 2.0 ** -125
INF = float("inf")


def CHAIN(V):
    return 64 + V / 128


def _np(t):
    return t.detach().double().cpu().numpy()


def _half_step(want, dtype):
    f = torch.finfo(dtype)
    return np.abs(want) * f.eps / 2 + f.smallest_normal * f.eps / 2


def _near(got, want, bound, label=""):
    got = _np(got)
    assert got.shape == want.shape, f"{label}: {got.shape} != {want.shape}"
    with np.errstate(invalid="ignore"):
        want = np.where(np.abs(want) > torch.finfo(F32).max, np.sign(want) * np.inf, want)  # (float32 has no such number)
        good = (np.abs(got - want) <= bound) | (got == want) | (np.isnan(got) & np.isnan(want))
    if not good.all():
        i = tuple(np.argwhere(~good)[0])
        raise AssertionError(f"{label}: {int((~good).sum())} of {good.size} out of tolerance, first at {i}: got {got[i]}, "
                             f"want {want[i]}, bound {np.broadcast_to(bound, got.shape)[i]}")


def _logits(T, V, dtype, seed, kind="plain"):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn((T, V), generator=g) * 3
    if kind == "ties":
        l = torch.randint(-2, 3, (T, V), generator=g).float() * 0.5
        l[l == 0] = torch.where(torch.rand(int((l == 0).sum()), generator=g) < 0.5, 0.0, -0.0)
    if kind == "masked":
        l[torch.rand((T, V), generator=g) < 0.7] = -INF
        l[0] = -INF
        l[-1, 1:] = -INF
    if kind == "lowest":
        l[torch.rand((T, V), generator=g) < 0.5] = torch.finfo(dtype).min
        l[0] = torch.finfo(dtype).min
    if kind == "peaked":
        l = l * 10
        l[:, V // 2] += 40
    if kind == "equal":
        l[:] = 1.5
    if kind == "rising":
        l = torch.linspace(-9, 9, V).repeat(T, 1)
    if kind == "falling":
        l = torch.linspace(9, -9, V).repeat(T, 1)
    return l.to(dtype).to(DEV)


class Bounds:
    """What every value of a matrix of logits may be off by."""

    def __init__(self, x, scale):
        T, V = x.shape
        with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
            m = x.max(1, keepdims=True)
            some = m > -np.inf
            self.d = np.where(x > -np.inf, scale * (np.where(some, m, 0) - x), 0)
            e = np.where(x > -np.inf, np.exp(-self.d), 0)
            S = np.where(some[:, 0], e.sum(1), 1)
            self.p = e / S[:, None]
            self.log_S = np.log(S)
            d = np.minimum(self.d, 104)
            self.mean_d = (self.p * d).sum(1)
            self.S = U * (2.5 * self.mean_d + 4 * CHAIN(V) + 8)  # relative
            self.term = U * (2.5 * d + 8) + self.S[:, None]      # of p, relative
            self.H = U * ((self.p * d * (2.5 * d + 4 * CHAIN(V) + 12)).sum(1) + 2 * self.log_S + self.log_S + self.mean_d) \
                + self.S * (1 + self.mean_d)
        self.m, self.scale = m[:, 0], scale

    def logprob(self, at):
        """at: (T, j) indices, -1 for none."""
        d = np.take_along_axis(self.d, np.maximum(at, 0), 1)
        return U * (3.5 * np.minimum(d, 1e38) + 3 * self.log_S[:, None]) + self.S[:, None] + TINY

    def lse(self):
        with np.errstate(invalid="ignore"):
            return U * (np.abs(self.scale * self.m) + 4 * self.log_S) + self.S

    def gradient(self, marked, size, of_entropy, entropy, want, dtype):
        """size: (T,) sum of the magnitudes of what multiplies p; of_entropy (T,);
        marked (T, V): sum of magnitudes of what is added at a token."""
        n = 80
        reach = self.d + np.abs(entropy)[:, None] + self.log_S[:, None]
        reach = np.minimum(reach, 1e30)
        slip = self.p * ((self.term + n * U) * size[:, None]
                         + np.abs(of_entropy)[:, None] * ((self.term + n * U) * reach + self.H[:, None]))
        small = TINY * (size + 400 * np.abs(of_entropy))[:, None]
        return self.scale * (slip + n * U * marked + small) + (1 + 4 * U) * _half_step(want, dtype) + 2 * U * np.abs(want)


SIZES = [(1, 1), (3, 2), (5, 3), (4, 7), (3, 31), (5, 64), (4, 65), (9, 118), (3, 255), (4, 256), (2, 257), (3, 511),
         (3, 513), (3, 1000), (2, 2048), (2, 2049), (2, 4096), (2, 4097), (2, 8195), (1, 32003)]


def _check_logprobs(x, ids, k, scale, label, gradients=True):
    T, V = x.shape
    dtype = x.dtype
    host, hids = _np(x), ids.cpu().numpy()
    want = ref.logprobs_ref(host, hids, k, scale)
    r = lg.logprobs_forward(x, ids, k, scale, entropy=True)
    b = Bounds(host, scale)
    for t in (r.logprob, r.lse, r.entropy, r.stats):
        assert t.dtype == F32
    at = np.where((hids >= 0) & (hids < V), hids, 0)[:, None]
    _near(r.logprob, want["logprob"], b.logprob(at)[:, 0], label + " logprob")
    _near(r.lse, want["lse"], b.lse(), label + " lse")
    _near(r.entropy, want["entropy"], b.H + U, label + " entropy")
    if k:
        assert r.top_ids.dtype == torch.int32
        assert np.array_equal(r.top_ids.cpu().numpy(), want["top_ids"]), label + " top ids"
        _near(r.top, want["top"], b.logprob(want["top_ids"]), label + " top")
    else:
        assert r.top is None and r.top_ids is None
    if not gradients:
        return
    rng = np.random.default_rng(T + V + k)
    g = dict(grad_logprob=rng.normal(size=T), grad_lse=rng.normal(size=T), grad_entropy=rng.normal(size=T))
    if k:
        g["grad_top"] = rng.normal(size=(T, k))
    g = {n: v.astype(np.float32) for n, v in g.items()}
    up = {n: torch.from_numpy(v).to(DEV) for n, v in g.items()}
    inside = (hids >= 0) & (hids < V)
    for names in (["grad_logprob"], ["grad_lse", "grad_entropy"], ["grad_top"], list(g)):
        if any(n not in g for n in names):
            continue
        grad = lg.logprobs_backward(x, r, ids, scale, **{n: up[n] for n in names})
        assert grad.dtype == dtype and grad.shape == x.shape
        wanted = ref.logprobs_backward_ref(host, hids, want["top_ids"], scale, **{n: g[n].astype(np.float64) for n in names})
        marked, size, gh = np.zeros((T, V)), np.zeros(T), np.zeros(T)
        if "grad_logprob" in names:
            own = np.where(inside, np.abs(g["grad_logprob"]), 0)
            np.add.at(marked, (np.arange(T), at[:, 0]), own)
            size += own
        if "grad_lse" in names:
            size += np.abs(g["grad_lse"])
        if "grad_top" in names:
            own = np.where(want["top_ids"] >= 0, np.abs(g["grad_top"]), 0)
            np.add.at(marked, (np.arange(T)[:, None], np.maximum(want["top_ids"], 0)), own)
            size += own.sum(1)
        if "grad_entropy" in names:
            gh = g["grad_entropy"]
        _near(grad, wanted, b.gradient(marked, size, gh, want["entropy"], wanted, dtype), f"{label} gradient {names}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", SIZES)
def test_logprobs(T, V, dtype):
    say(f"logprobs T={T} V={V} {dtype}")
    for i, kind in enumerate(("plain", "ties", "masked", "lowest", "peaked")):
        rng = np.random.default_rng(V + i)
        ids = torch.from_numpy(rng.integers(-1, V + 1, T)).to([torch.int32, torch.int64][i % 2]).to(DEV)
        k = min(V, [0, 1, 5, 20, 64][(V + i) % 5])
        _check_logprobs(_logits(T, V, dtype, T * V, kind), ids, k, [1.0, 0.37, 2.5][(i + T) % 3], f"{kind} k={k}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,k", [(3, 50021, 50), (2, 131072, 20), (1, 262147, 64), (1, 1 << 20, 7), (70, 9001, 3)])
def test_logprobs_long_rows(T, V, k, dtype):
    say(f"logprobs T={T} V={V} k={k} {dtype}")
    ids = torch.from_numpy(np.random.default_rng(V).integers(0, V, T)).to(DEV)
    for kind in ("plain", "masked") if T * V < 1 << 19 else ("plain",):
        _check_logprobs(_logits(T, V, dtype, V, kind), ids, k, 1.0, kind, gradients=T * V < 1 << 19)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [4111, 16391, 50021])
def test_tokens_at_a_rows_ends(V, dtype):
    """Given tokens among the elements before a row's first whole cache line and behind its last whole vector, in rows
    that begin at every place of a line."""
    T = 13
    say(f"ends V={V} {dtype}")
    x = _logits(T, V, dtype, V)
    for ids in ([0] * T, [V - 1] * T, [(5 * t) % 64 for t in range(T)], [V - 1 - t % 8 for t in range(T)]):
        _check_logprobs(x, torch.tensor(ids, device=DEV), 2, 1.0, "ends")


@pytest.mark.parametrize("k", [1, 2, 16, 17, 40, 63, 64])
@pytest.mark.parametrize("V", [64, 118, 300, 1000, 5000, 40000])
def test_alternatives(V, k):
    """Choices whatever the order and the ties of a row (T of few and of many rows)."""
    say(f"alternatives V={V} k={k}")
    for dtype in TYPES:
        for kind in ("plain", "ties", "equal", "rising", "falling", "masked", "peaked"):
            for T in (2, 5):
                x = _logits(T, V, dtype, V + k, kind)
                r = lg.logprobs_forward(x, k=k)
                l = x.float().cpu()
                best, at = torch.sort(l, dim=1, descending=True, stable=True)
                at = torch.where(best > -INF, at, -1)[:, :k]
                assert torch.equal(r.top_ids.cpu().long(), at), f"{dtype} {kind} T={T}"
                assert r.logprob is None and r.entropy is None
                lp = torch.log_softmax(l.double(), 1)
                on = at >= 0
                want = lp.gather(1, at.clamp_min(0))
                assert (torch.where(on, (r.top.cpu().double() - want).abs(), 0.0) < 1e-4).all()
                assert (r.top.cpu()[~on] == -INF).all()


def test_few_tokens_allowed():
    """Constrained decoding: fewer finite logits than alternatives, anywhere in a long row."""
    for V in (100, 3000, 70000, 200001):
        for dtype in TYPES:
            x = torch.full((4, V), -INF, dtype=dtype, device=DEV)
            places = [[V - 1], [0, V // 2], list(range(min(V, 40))), list(range(V - 30, V))]
            for t, p in enumerate(places):
                x[t, p] = torch.linspace(0, 3, len(p), device=DEV).to(dtype)
            r = lg.logprobs_forward(x, torch.tensor([V - 1, 0, 1, V], device=DEV), k=50)
            for t, p in enumerate(places):
                order = sorted(p, key=lambda v: (-float(x[t, v]), v))
                assert r.top_ids[t].tolist() == (order + [-1] * 50)[:50]
                assert abs(float(r.top[t].exp().sum()) - 1) < 1e-5
            assert r.logprob[0] == 0 and r.logprob[3] == 0


def test_rows_without_a_distribution():
    nan = float("nan")
    for V in (6, 400, 6000, 300000):
        x = torch.zeros((6, V), device=DEV)
        x[0] = -INF
        x[1, V // 3] = nan
        x[2, 1] = INF
        x[3, 5:] = -INF
        x[4] = nan
        ids = torch.tensor([1, 2, 0, V - 1, -1, 0], device=DEV)
        r = lg.logprobs_forward(x, ids, 3, 1.0, True)
        assert r.logprob[0] == -INF and r.lse[0] == -INF and r.entropy[0] == 0
        assert r.top_ids[0].tolist() == [-1] * 3 and (r.top[0] == -INF).all()
        for t in (1, 2, 4):
            assert torch.isnan(r.lse[t]) and torch.isnan(r.entropy[t]) and torch.isnan(r.top[t]).all()
        assert torch.isnan(r.logprob[1:3]).all() and r.logprob[4] == 0
        assert r.top_ids[1].tolist() == [v for v in range(4) if v != V // 3][:3]
        assert r.top_ids[2].tolist() == [1, 0, 2] and r.top_ids[4].tolist() == [-1] * 3
        # (a barred token: no probability; the rest share it)
        assert r.logprob[3] == (0 if V <= 5 else -INF) and abs(float(r.lse[3]) - np.log(5)) < 1e-6
        g = torch.ones(6, device=DEV)
        grad = lg.logprobs_backward(x, r, ids, grad_logprob=g, grad_entropy=g, grad_top=torch.ones(6, 3, device=DEV))
        assert not grad[0].any() and torch.isnan(grad[1]).all() and torch.isfinite(grad[[3, 5]]).all()
        # padding: rows of dropped ids are zeros whatever they hold
        pad = torch.full((6,), -1, device=DEV)
        assert not lg.logprobs_backward(x, r, pad, grad_logprob=g).any()
        assert not lg.logprobs_backward(x, r, ids, grad_logprob=0 * g, grad_lse=0 * g).any()
        assert torch.isnan(lg.logprobs_backward(x, r, ids, grad_logprob=nan * g)[[1, 2, 3, 5]]).all()
        # distillation from token 0 (kept), or from nothing
        t = torch.zeros(6, 2, device=DEV)
        kept = torch.tensor([[0, -1]], dtype=torch.int32, device=DEV).repeat(6, 1)
        for call in (lambda i: lg.distill_step(g, x, i, t), lambda i: _two_calls(g, x, i, t, 1.0, True)):
            loss, grad = call(kept)
            assert loss[0] == INF and torch.isnan(loss[[1, 2, 4]]).all() and torch.isfinite(loss[[3, 5]]).all()
            assert not grad[0].any() and torch.isnan(grad[[1, 4]]).all() and torch.isfinite(grad[[3, 5]]).all()
            loss, grad = call(torch.full_like(kept, V))
            assert not loss.any() and not grad.any()


# -------------------------------------------------------------- distillation

def _two_calls(g, x, ids, teacher, scale, renormalise):
    loss, stats = lg.distill_forward(x, ids, teacher, scale, renormalise)
    return loss, lg.distill_backward(g, x, ids, teacher, stats, scale, renormalise)


def _check_distill(x, ids, teacher, scale, renormalise, label, g=None):
    T, V = x.shape
    k = ids.shape[1]
    host, hids, ht = _np(x), ids.cpu().numpy(), _np(teacher)
    if g is None:
        g = torch.randn(T, generator=torch.Generator().manual_seed(V)).to(DEV)
    want = ref.distill_ref(host, hids, ht, scale, renormalise)
    wanted = ref.distill_backward_ref(_np(g), host, hids, ht, scale, renormalise)
    b = Bounds(host, scale)
    bound, marked, size = np.zeros(T), np.zeros((T, V)), np.zeros(T)
    for t in range(T):
        kept, logq = ref.taught(hids[t], ht[t], V, renormalise)
        if not kept:
            continue
        q = np.exp(logq)
        at = hids[t][kept]
        # log q: the slot's log probability, the row's largest and the log of their sum are rounded and subtracted
        off = U * (3 * np.abs(ht[t][kept]) + 3 * np.abs(logq) + (k + 16 if renormalise else 0))
        lp, _ = ref.distribution(host[t], scale)
        diff = np.abs(np.where(q > 0, logq - lp[at], 0))
        own = b.logprob(np.broadcast_to(at, (T, len(at))))[t]
        with np.errstate(invalid="ignore"):
            bound[t] = (q * ((off + (k + 8) * U) * np.where(np.isfinite(diff), diff, 0) + off + own)).sum() + TINY
        slip = q * (off + (k + 8) * U) / (80 * U)  # (in units of what Bounds.gradient allows for)
        np.add.at(marked[t], at, (q + slip) * abs(float(g[t])))
        size[t] = (q + slip).sum() * abs(float(g[t]))
    bound += 2 * U * np.abs(np.where(np.isfinite(want), want, 0))
    allowed = b.gradient(marked, size, np.zeros(T), np.zeros(T), wanted, x.dtype)
    for name, call in (("two calls", lambda: _two_calls(g, x, ids, teacher, scale, renormalise)),
                       ("step", lambda: lg.distill_step(g, x, ids, teacher, scale, renormalise))):
        loss, grad = call()
        assert loss.dtype == F32 and grad.dtype == x.dtype
        _near(loss, want, bound, f"{label} {name} loss")
        _near(grad, wanted, allowed, f"{label} {name} gradient")


def _teacher(T, V, k, seed, kind="plain"):
    """k different tokens a row (or the same ones again), and log probabilities that sum to less than 1."""
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.permutation(V)[:k] if V >= k else rng.integers(0, V, k) for _ in range(T)])
    t = np.log(rng.dirichlet(np.ones(k + 1), size=T)[:, :k]) if k > 0 else np.zeros((T, 0))
    if kind == "holes":
        ids[rng.random(ids.shape) < 0.3] = -1
        ids[rng.random(ids.shape) < 0.1] = V
        t[rng.random(t.shape) < 0.2] = -np.inf
        ids[0] = -1
    if kind == "again":
        ids[:, : (k + 1) // 2] = ids[:, :1]
    return torch.from_numpy(ids), torch.from_numpy(t.astype(np.float32)).to(DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", SIZES + [(3, 20011), (2, 50021), (2, 131072), (1, 200003), (1, 300007)])
def test_distill(T, V, dtype):
    say(f"distill T={T} V={V} {dtype}")
    for i, (kind, how) in enumerate((("plain", "plain"), ("ties", "holes"), ("masked", "holes"), ("lowest", "again"),
                                     ("peaked", "plain"))):
        if T * V > 1 << 18 and i % 2:
            continue
        k = min(V, [1, 3, 16, 64, 200][(V + i) % 5])
        ids, teacher = _teacher(T, V, k, V + i, how)
        ids = ids.to([torch.int32, torch.int64][i % 2]).to(DEV)
        x = _logits(T, V, dtype, T + V, kind)
        _check_distill(x, ids, teacher, [1.0, 0.5, 1.7][(i + V) % 3], i % 2 == 0, f"{kind} {how} k={k}")


def test_distill_zero_gradients_and_many_rows():
    """Rows without an outgoing gradient, among more rows than are in flight together."""
    T, V, k = 5000, 118, 8
    x = _logits(T, V, F32, 1)
    ids, teacher = _teacher(T, V, k, 2, "holes")
    ids = ids.to(torch.int32).to(DEV)
    g = torch.randn(T, device=DEV)
    g[::3] = 0
    x[::6] = float("nan")
    loss, grad = lg.distill_step(g, x, ids, teacher, 0.7)
    l2, g2 = _two_calls(g, x, ids, teacher, 0.7, True)
    assert not grad[::3].any() and not g2[::3].any()
    on = torch.ones(T, dtype=torch.bool, device=DEV)
    on[::6] = False
    lp = torch.log_softmax(x.double() * 0.7, 1)
    inside = (ids >= 0) & (ids < V) & (teacher > -INF)
    q = torch.softmax(torch.where(inside, teacher.double(), -INF), 1)
    q = torch.where(inside.any(1, keepdim=True), q, 0.0)
    want = torch.where(q > 0, q * (q.log() - lp.gather(1, ids.clamp(0, V - 1).long())), 0.0).sum(1)
    target = torch.zeros_like(lp).scatter_add_(1, ids.clamp(0, V - 1).long(), q)
    wanted = 0.7 * g.double()[:, None] * (q.sum(1, keepdim=True) * lp.exp() - target)
    wanted[~inside.any(1)] = 0
    for a, b in ((loss, grad), (l2, g2)):
        assert ((a - want)[on].abs() < 1e-5).all()
        assert ((b - wanted)[on].abs() < 1e-6 * g.abs()[on, None].double() + 1e-9).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [64, 118, 255, 300, 511, 2000])
def test_distill_of_short_rows_with_many_alternatives(V, dtype):
    for k in (15, 16, 17, 33, 63, 64, 65, 100, 256):
        if k > V:
            continue
        for how in ("plain", "holes", "again"):
            ids, teacher = _teacher(19, V, k, V + k, how)
            _check_distill(_logits(19, V, dtype, V), ids.to(DEV), teacher, 1.0, k % 2 == 0, f"{how} k={k}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V,k", [(1100, 4201, 5), (1500, 9003, 200), (1300, 20001, 64), (1200, 33001, 256), (600, 66000, 17),
                                   (520, 70003, 100), (513, 131072, 64)])
def test_distill_step_of_many_long_rows(T, V, k, dtype):
    """Rows that workgroups take one after the other, with repeated and dropped alternatives: against float64 on the
    device, under the bounds of this file's head for rows whose logits lie within 40 of their largest, with
    probabilities of at most 1."""
    if dtype == F32 and V > 70000:
        V = 65536 + 3
    say(f"distill step T={T} V={V} k={k} {dtype}")
    g = torch.Generator(device=DEV).manual_seed(T)
    x = (torch.randn((T, V), generator=g, device=DEV) * 2).to(dtype)
    ids = torch.randint(-V // 20, V + V // 20, (T, k), generator=g, device=DEV)
    ids[:, 0] = V - 1                       # behind the last whole vector
    ids[1::2, -1] = ids[1::2, 0]            # twice
    ids[::7] = -1
    teacher = torch.log_softmax(torch.randn((T, k), generator=g, device=DEV), 1)
    go = torch.randn(T, generator=g, device=DEV)
    go[3::11] = 0
    loss, grad = lg.distill_step(go, x, ids, teacher, 0.9)
    inside = (ids >= 0) & (ids < V)
    some = inside.any(1)
    q = torch.softmax(torch.where(inside, teacher.double(), -INF), 1)
    q = torch.where(some[:, None] & inside, q, 0.0)
    at = torch.where(inside, ids, 0)
    rel = U * (2.5 * 40 + 4 * CHAIN(V) + 2 * k + 60)
    half = torch.finfo(dtype).eps / 2
    for a in range(0, T, 64):
        b = min(a + 64, T)
        lp = torch.log_softmax(0.9 * x[a:b].double(), 1)
        want = torch.where(q[a:b] > 0, q[a:b] * (q[a:b].log() - lp.gather(1, at[a:b])), 0.0).sum(1)
        assert ((loss[a:b] - want).abs() <= rel * (1 + want.abs())).all()
        marks = torch.zeros_like(lp).scatter_add_(1, at[a:b], q[a:b])
        p = lp.exp() * some[a:b, None]
        wanted = 0.9 * go[a:b, None].double() * (p - marks)
        bound = 0.9 * go[a:b, None].abs().double() * rel * (p + marks) + wanted.abs() * half + torch.finfo(dtype).smallest_normal
        assert ((grad[a:b].double() - wanted).abs() <= bound * 1.001).all()
        assert not grad[a:b][~some[a:b] | (go[a:b] == 0)].any()


# ------------------------------------------------------------- shapes, places

def test_strided_and_expanded_rows():
    for dtype in TYPES:
        for V in (90, 3001, 40003):
            wide = _logits(5, V + 13, dtype, V)
            x = wide[:, 7:7 + V]
            ids = torch.tensor([0, V - 1, 3, -1, 5], device=DEV)
            tids, teacher = _teacher(5, V, 6, 1)
            tids = tids.to(DEV)
            g = torch.randn(5, device=DEV)
            for a in (x, x[:1].expand(5, V)):
                b = a.contiguous()
                p, q = (lg.logprobs_forward(z, ids, 9, 1.3, True) for z in (a, b))
                for n in ("logprob", "lse", "entropy", "top", "top_ids", "stats"):
                    assert torch.equal(getattr(p, n), getattr(q, n)), n
                assert torch.equal(lg.logprobs_backward(a, p, ids, 1.3, g, None, g), lg.logprobs_backward(b, p, ids, 1.3, g, None, g))
                for u, v in zip(lg.distill_step(g, a, tids, teacher), lg.distill_step(g, b, tids, teacher)):
                    assert torch.equal(u, v)
                for u, v in zip(_two_calls(g, a, tids, teacher, 1.0, False), _two_calls(g, b, tids, teacher, 1.0, False)):
                    assert torch.equal(u, v)


def test_no_rows_and_far_ids():
    x = torch.empty((0, 50), device=DEV)
    r = lg.logprobs_forward(x, torch.empty(0, dtype=torch.int64, device=DEV), 4, 1.0, True)
    assert r.top.shape == (0, 4) and r.logprob.shape == (0,)
    assert lg.logprobs_backward(x, r, grad_lse=r.lse).shape == (0, 50)
    i, t = torch.empty((0, 3), dtype=torch.int32, device=DEV), torch.empty((0, 3), device=DEV)
    loss, grad = lg.distill_step(r.lse, x, i, t)
    assert loss.shape == (0,) and grad.shape == (0, 50)
    far = torch.tensor([1 << 32, (1 << 32) + 1, -(1 << 63), (1 << 63) - 1, 50, -1], device=DEV)
    x = _logits(6, 50, F32, 0)
    r = lg.logprobs_forward(x, far)
    assert not r.logprob.any()
    assert not lg.logprobs_backward(x, r, far, grad_logprob=torch.ones(6, device=DEV)).any()
    assert not lg.distill_forward(x, far[:, None], torch.zeros(6, 1, device=DEV))[0].any()


def test_places_past_32_bits():
    """Rows that lie more than 2^32 elements into their matrices."""
    T, V = (1 << 17) + 5, 32781  # 4.3e9 elements, 8.6 GB
    x = torch.zeros((T, V), dtype=BF16, device=DEV)
    x[-1] = _logits(1, V, BF16, 4)[0]
    ids = torch.full((T,), -1, device=DEV)
    ids[-1] = 77
    r = lg.logprobs_forward(x, ids, 2)
    one = lg.logprobs_forward(x[-1:], ids[-1:], 2)
    assert torch.equal(r.logprob[-1:], one.logprob) and torch.equal(r.top_ids[-1:], one.top_ids)
    assert torch.equal(r.lse[-1:], one.lse) and abs(float(r.lse[0]) - np.log(V)) < 1e-5
    g = torch.ones(T, device=DEV)
    grad = lg.logprobs_backward(x, r, ids, grad_logprob=g)
    assert torch.equal(grad[-1:], lg.logprobs_backward(x[-1:], one, ids[-1:], grad_logprob=g[-1:]))
    assert not grad[:-1].any()
    del grad
    tids = torch.full((T, 2), -1, device=DEV)
    tids[-1] = torch.tensor([5, V - 1])
    t = torch.zeros((T, 2), device=DEV)
    loss, grad = lg.distill_step(g, x, tids, t)
    l1, g1 = lg.distill_step(g[-1:], x[-1:], tids[-1:], t[-1:])
    # (one row may be formed by another split of the sums)
    assert abs(float(loss[-1] - l1[0])) < 1e-5 and torch.allclose(grad[-1].float(), g1[0].float(), rtol=1e-2, atol=1e-8)
    assert not grad[:-1].any() and not loss[:-1].any()


def test_the_same_call_twice_gives_the_same_bits():
    for T, V in ((300, 118), (2, 100003), (40, 20000)):
        x = _logits(T, V, BF16, 3)
        ids = torch.randint(0, V, (T,), device=DEV)
        tids, teacher = _teacher(T, V, 30, 1)
        tids, g = tids.to(DEV), torch.randn(T, device=DEV)
        a, b = (lg.logprobs_forward(x, ids, 30, 1.0, True) for _ in range(2))
        for n in ("logprob", "lse", "entropy", "top", "top_ids", "stats"):
            assert torch.equal(getattr(a, n), getattr(b, n))
        for u, v in zip(lg.distill_step(g, x, tids, teacher), lg.distill_step(g, x, tids, teacher)):
            assert torch.equal(u, v)


# ------------------------------------------------------ streams, graphs, autograd

def test_other_stream():
    T, V = 30, 9001
    x = _logits(T, V, BF16, 0)
    ids = torch.randint(0, V, (T,), device=DEV)
    tids, teacher = _teacher(T, V, 8, 0)
    tids, g = tids.to(DEV), torch.randn(T, device=DEV)
    r = lg.logprobs_forward(x, ids, 5)
    want = [r.logprob, r.top, lg.logprobs_backward(x, r, ids, grad_logprob=g), *_two_calls(g, x, tids, teacher, 1.0, True),
            *lg.distill_step(g, x, tids, teacher)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    r = lg.logprobs_forward(x, ids, 5, stream=s)
    loss, stats = lg.distill_forward(x, tids, teacher, stream=s)
    got = [r.logprob, r.top, lg.logprobs_backward(x, r, ids, grad_logprob=g, stream=s), loss,
           lg.distill_backward(g, x, tids, teacher, stats, stream=s), *lg.distill_step(g, x, tids, teacher, stream=s.cuda_stream)]
    s.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_two_streams_at_once():
    """Calls of two streams in flight together share nothing."""
    T, V, k = 3, 200003, 9
    xs = [_logits(T, V, BF16, i) for i in range(2)]
    ids = torch.randint(0, V, (T,), device=DEV)
    tids, teacher = _teacher(T, V, k, 0)
    tids, g = tids.to(DEV), torch.randn(T, device=DEV)

    def calls(x):
        r = lg.logprobs_forward(x, ids, k)
        return [r.logprob, r.top, r.top_ids, *_two_calls(g, x, tids, teacher, 1.0, True)]

    want = [calls(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(calls(xs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for one in got[i]:
            for a, b in zip(one, want[i]):
                assert torch.equal(a, b)


def test_graph_replays():
    """Captured calls on changed inputs; two graphs have workspaces of their own."""
    T, V, k = 4, 120001, 12
    x = _logits(T, V, F16, 0)
    ids = torch.randint(0, V, (T,), device=DEV)
    tids, teacher = _teacher(T, V, k, 0)
    tids, g = tids.to(DEV), torch.randn(T, device=DEV)

    def calls():
        r = lg.logprobs_forward(x, ids, k, 1.1, True)
        return [r.logprob, r.entropy, r.top, r.top_ids, lg.logprobs_backward(x, r, ids, 1.1, g, None, g, r.top),
                *_two_calls(g, x, tids, teacher, 1.1, True), *lg.distill_step(g, x, tids, teacher, 1.1)]

    calls()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = calls()
        graphs.append((graph, out))
    for i in range(4):
        x.copy_(_logits(T, V, F16, 10 + i, ["plain", "masked"][i % 2]))
        ids.copy_(torch.randint(0, V, (T,), device=DEV))
        want = [w.clone() for w in calls()]
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for a, b in zip(out, want):
                assert torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float()))


def test_autograd():
    T, V, k = 6, 300, 5
    x = _logits(T, V, F32, 0).requires_grad_()
    ids = torch.tensor([3, -1, 299, 0, 7, 300], device=DEV)
    r = lg.logprobs(x, ids, k, 0.8, True)
    assert not r.top_ids.requires_grad and not r.stats.requires_grad
    w = torch.randn(T, k, device=DEV)
    (r.logprob.sum() + 2 * r.entropy.sum() + (w * r.top).sum() + (r.lse ** 2).sum()).backward()
    y = x.detach().double().requires_grad_()
    lp = torch.log_softmax(0.8 * y, 1)
    inside = (ids >= 0) & (ids < V)
    total = torch.where(inside, lp.gather(1, ids.clamp(0, V - 1)[:, None])[:, 0], 0.0).sum()
    total = total - 2 * (lp.exp() * lp).sum() + (w * lp.gather(1, r.top_ids.long())).sum() \
        + (torch.logsumexp(0.8 * y, 1) ** 2).sum()
    total.backward()
    assert (x.grad.double() - y.grad).abs().max() < 1e-4
    # one value only; and an answer taught to a student
    x.grad = None
    lg.logprobs(x, ids).logprob.sum().backward()
    assert x.grad.shape == x.shape
    student = _logits(T, V, BF16, 5).requires_grad_()
    with torch.no_grad():
        answer = lg.logprobs(x, k=k)
    loss = lg.distill(student, answer.top_ids, answer.top, 1.5, False)
    (loss * torch.arange(6, device=DEV)).sum().backward()
    g = torch.arange(6, device=DEV).float()
    want = ref.distill_backward_ref(_np(g), _np(student), answer.top_ids.cpu().numpy(), _np(answer.top), 1.5, False)
    assert np.abs(_np(student.grad) - want).max() < 0.05
    assert torch.equal(student.grad, lg.distill_step(g, student.detach(), answer.top_ids, answer.top, 1.5, False)[1])
    assert lg.distill(student.detach(), answer.top_ids, answer.top).requires_grad is False


def test_gradients_are_differences():
    """Directional differences of the kernels' own losses, in float32: with a step h of 2^-7, third derivatives
    (below 4 here) leave 4 h^2 / 6, roundings of the two losses (6 values up to 16) 2^-20 / h."""
    T, V, k, h = 6, 200, 7, 2.0 ** -7
    x = _logits(T, V, F32, 2) * 0.3
    ids = torch.randint(0, V, (T,), device=DEV)
    tids, teacher = _teacher(T, V, k, 1)
    tids = tids.to(DEV)
    one = torch.ones(T, device=DEV)
    g = torch.Generator().manual_seed(5)
    for _ in range(4):
        d = torch.randn((T, V), generator=g).to(DEV)
        d /= d.norm(dim=1, keepdim=True)
        up, down = (lg.logprobs_forward(x + s * h * d, ids, 0, 1.0, True) for s in (1, -1))
        r = lg.logprobs_forward(x, ids, 0, 1.0, True)
        grad = lg.logprobs_backward(x, r, ids, 1.0, one, None, one)
        diff = (up.logprob - down.logprob + up.entropy - down.entropy) / (2 * h)
        assert ((grad * d).sum(1) - diff).abs().max() < 4 * h * h / 6 + 2.0 ** -20 / h
        loss = [lg.distill_forward(x + s * h * d, tids, teacher)[0] for s in (1, -1)]
        grad = lg.distill_step(one, x, tids, teacher)[1]
        assert ((grad * d).sum(1) - (loss[0] - loss[1]) / (2 * h)).abs().max() < 4 * h * h / 6 + 2.0 ** -20 / h


def test_captured_backward():
    """Forward and backward of the differentiable forms as one graph, with no other graph of the leaf alive."""
    T, V = 8, 1500
    x = _logits(T, V, F32, 0).requires_grad_()
    ids = torch.randint(0, V, (T,), device=DEV)
    tids, teacher = _teacher(T, V, 4, 0)
    tids = tids.to(DEV)

    def step():
        x.grad = None
        r = lg.logprobs(x, ids, entropy=True)
        (r.logprob.sum() + r.entropy.sum() + lg.distill(x, tids, teacher).sum()).backward()

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    x.grad = None
    with torch.cuda.graph(graph):
        step()
    captured = x.grad
    for i in range(3):
        with torch.no_grad():
            x.copy_(_logits(T, V, F32, 20 + i))
        graph.replay()
        torch.cuda.synchronize()
        got = captured.clone()
        y = x.detach().clone().requires_grad_()
        r = lg.logprobs(y, ids, entropy=True)
        (r.logprob.sum() + r.entropy.sum() + lg.distill(y, tids, teacher).sum()).backward()
        assert torch.equal(got, y.grad)


def test_refusals():
    x = _logits(4, 50, F32, 0)
    ids = torch.zeros(4, dtype=torch.int64, device=DEV)
    r = lg.logprobs_forward(x, ids, 3)
    g = torch.ones(4, device=DEV)
    tids, t = torch.zeros((4, 2), dtype=torch.int32, device=DEV), torch.zeros((4, 2), device=DEV)
    bad = [lambda: lg.logprobs_forward(x.double(), ids), lambda: lg.logprobs_forward(x.t(), ids),
           lambda: lg.logprobs_forward(x, ids[:3]), lambda: lg.logprobs_forward(x, ids.float()),
           lambda: lg.logprobs_forward(x, ids.cpu()), lambda: lg.logprobs_forward(x, k=-1),
           lambda: lg.logprobs_forward(x, k=1 << 32), lambda: lg.logprobs_forward(x[0]),
           lambda: lg.logprobs_backward(x, r, grad_logprob=g), lambda: lg.logprobs_backward(x, r, ids, grad_entropy=g),
           lambda: lg.logprobs_backward(x, lg.logprobs_forward(x), grad_top=t),
           lambda: lg.logprobs_backward(x, r, ids, grad_logprob=g.double()),
           lambda: lg.logprobs_backward(x, r, ids, grad_top=t), lambda: lg.logprobs_backward(x[:3], r, grad_lse=g[:3]),
           lambda: lg.distill_forward(x, tids, t[:, :1]), lambda: lg.distill_forward(x, tids[:3], t[:3]),
           lambda: lg.distill_forward(x, tids, t.to(F16)), lambda: lg.distill_step(g[:2], x, tids, t),
           lambda: lg.distill_backward(g, x, tids, t, r.stats[:, :1])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    from paper_2211_17111_amd import BevpoolError
    for call in (lambda: lg.logprobs_forward(x, k=51), lambda: lg.logprobs_forward(x, ids, scale=0.0),
                 lambda: lg.distill_forward(x, tids[:, :0], t[:, :0]), lambda: lg.distill_forward(x, tids, t, INF)):
        with pytest.raises(BevpoolError):
            call()
    with torch.autograd.graph.saved_tensors_hooks(lambda a: a, lambda a: a[..., :1] if a.dim() == 2 else a):
        y = x.clone().requires_grad_()
        loss = lg.distill(y, tids, t).sum()
        p = lg.logprobs(y, ids).logprob.sum()
    for v in (loss, p):
        with pytest.raises(ValueError):
            v.backward()


def test_distil_an_expert_model():
    """The operators as they are used together: a teacher's layer of experts answers for a few tokens, and its
    alternatives teach a student, whose table and layer receive gradients."""
    T, V, C, E, k, F = 24, 700, 64, 8, 2, 96
    g = torch.Generator().manual_seed(0)

    def normal(*shape):
        return (torch.randn(shape, generator=g) * shape[-1] ** -0.5).to(DEV)

    ids = torch.randint(0, V, (T,), generator=g).to(DEV)
    table, router = normal(V, C), normal(C, E)
    up, down, head = normal(E, 2 * F, C), normal(E, C, F), normal(V, C) * 8
    x = rows.embed_forward(table, ids, C ** 0.5)
    weights, experts = rows.route_forward(x @ router, k)
    layer = rows.expert_layer_forward(x, up, down, weights, experts)
    # the same layer by dispatch, the experts one by one, and combine
    r, plan = rows.dispatch_forward(x, experts, E)
    y = torch.empty_like(r)
    offsets = plan.offsets.tolist()
    for e in range(E):
        mine = r[offsets[e]:offsets[e + 1]]
        y[offsets[e]:offsets[e + 1]] = (torch.nn.functional.silu(mine @ up[e, :F].t()) * (mine @ up[e, F:].t())) @ down[e].t()
    same = rows.combine_forward(y, weights, plan)
    assert (layer - same).abs().max() < 1e-4 * same.abs().max()
    answer = lg.logprobs_forward((x + layer) @ head.t(), k=16, entropy=True)
    want = torch.log_softmax(((x + layer) @ head.t()).double(), 1)
    assert (answer.top - torch.sort(want, 1, descending=True).values[:, :16]).abs().max() < 1e-4
    student_table, student_head = normal(V, C).requires_grad_(), normal(V, C).requires_grad_()
    loss = lg.distill(rows.embed(student_table, ids, C ** 0.5) @ student_head.t(), answer.top_ids, answer.top, 1.0, False)
    loss.mean().backward()
    a, b = (p.detach().double().requires_grad_() for p in (student_table, student_head))
    lp = torch.log_softmax(a[ids] * C ** 0.5 @ b.t(), 1).gather(1, answer.top_ids.long())
    plain = (answer.top.double().exp() * (answer.top.double() - lp)).sum(1)
    plain.mean().backward()
    assert (loss - plain).abs().max() < 1e-5
    for p, q in ((student_table, a), (student_head, b)):
        assert (p.grad - q.grad).abs().max() < 1e-5 * q.grad.abs().max()
