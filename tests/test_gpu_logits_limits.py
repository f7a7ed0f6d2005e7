"""Logits operators on the GPU at the ends of what they take."""

import numpy as np
import pytest
import torch

from _gpu import DEV, say
from paper_2211_17111_amd import logits as lg
from test_gpu_logits import CHAIN, F32, INF, TYPES, U, Bounds, _logits, _np, _two_calls

pytestmark = pytest.mark.gpu


def test_the_largest_scales():
    """All probability on the largest logits, shared by equal ones; nothing is NaN."""
    for V in (50, 3001, 40000, 300007):
        for dtype in TYPES:
            for scale in (2.0 ** 127, 2.35e38):
                x = torch.linspace(-4, 4, V, device=DEV).to(dtype).repeat(3, 1)
                x[0, 3], x[1, 7], x[1, V - 1] = 9, 9, 9
                x[2] = 1.5
                r = lg.logprobs_forward(x, torch.tensor([3, 7, 0], device=DEV), 2, scale, True)
                shares = torch.tensor([1.0, 2.0, V], dtype=torch.float64).log()
                for got, want in ((r.logprob, -shares), (r.entropy, shares), (r.top[:, 0], -shares)):
                    assert ((got.cpu().double() - want).abs() <= 2.0 ** -20 * (1 + want.abs())).all(), (V, dtype, scale)
                assert r.top_ids.tolist() == [[3, int(x[0].float().cpu().sort(descending=True, stable=True).indices[1])],
                                              [7, V - 1], [0, 1]]
                assert (r.top[0, 1], r.lse[0]) == (-INF, INF)
                ids = torch.tensor([[3, -1], [7, V - 1], [0, 1]], device=DEV)
                teacher = torch.zeros((3, 2), device=DEV)
                g = torch.full((3,), 0.5, device=DEV) / scale
                for loss, grad in (_two_calls(g, x, ids, teacher, scale, True), lg.distill_step(g, x, ids, teacher, scale)):
                    want = torch.tensor([0.0, 0.0, np.log(V / 2)], dtype=torch.float64)
                    assert ((loss.cpu().double() - want).abs() <= 2.0 ** -20 * (1 + want)).all()
                    assert torch.isfinite(grad).all() and (grad[:2].float().abs() < 1e-6).all()


def test_statistics():
    """Every row's largest logit and sum, whatever else is asked for: also where the largest is the type's lowest, a
    row holds a NaN or +inf, or nothing at all."""
    nan = float("nan")
    for V in (6, 118, 400, 3001, 9000, 40000, 300007):
        for dtype in TYPES:
            x = _logits(9, V, dtype, V, "masked" if V > 100 else "plain")
            x[0] = -INF
            x[1] = nan
            x[2], x[2, V // 2] = -INF, nan
            x[3, V - 1] = nan
            x[4, V // 3] = INF
            x[5], x[5, 1] = torch.finfo(dtype).min, -INF
            x[6], x[6, V // 2] = -INF, -2.5
            host = _np(x)
            m = np.where(np.isnan(host), -INF, host).max(1)
            whole = ~(np.isnan(host).any(1) | (host == INF).any(1))
            b = Bounds(host[whole], 0.7)
            with np.errstate(invalid="ignore"):
                S = np.where(host[whole] > -INF, np.exp(0.7 * (host[whole] - m[whole, None])), 0).sum(1)
            ids, teacher = torch.zeros((9, 2), dtype=torch.int32, device=DEV), torch.zeros((9, 2), device=DEV)
            few = min(20, V // 2)
            for stats in (lg.logprobs_forward(x, scale=0.7).stats, lg.logprobs_forward(x, None, 3, 0.7).stats,
                          lg.logprobs_forward(x, None, 6, 0.7, True).stats, lg.logprobs_forward(x, scale=0.7, entropy=True).stats,
                          lg.distill_forward(x, ids, teacher, 0.7)[1], lg.distill_forward(x, ids.repeat(1, few), teacher.repeat(1, few),
                                                                                          0.7)[1]):
                got = _np(stats)
                assert np.array_equal(got[:, 0], m), (V, dtype, got[:, 0], m)
                assert np.isnan(got[~whole, 1]).all()
                assert (np.abs(got[whole, 1] - S) <= b.S * S).all(), (V, dtype)


def _mixed(T, V, dtype, seed):
    """Rows of five kinds in turn: normal; 9 values only; equal; the best at a row's end; and at its beginning."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((T, V), generator=g, device=DEV) * 3
    x[1::5] = torch.randint(-4, 5, (len(range(1, T, 5)), V), generator=g, device=DEV).float() * 0.5
    x[2::5] = 1.5
    x[3::5] = torch.linspace(-9, 9, V, device=DEV)
    x[4::5] = torch.linspace(9, -9, V, device=DEV)
    x[7::10, : V // 2] = -INF
    return x.to(dtype)


@pytest.mark.parametrize("k", [1, 20, 64])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,batches,more", [(1030, 16, 0), (1030, 16, -1), (1030, 16, 1), (1030, 16, 8), (1030, 16, 4001), (1100, 5, 0),
                                            (1030, 8, 77), (1500, 11, 3), (400, 16, 0), (300, 40, 5), (1025, 33, 0)])
def test_alternatives_of_long_parts(T, batches, more, dtype, k):
    """Parts of 5 to 16 batches of 1024 vectors, the most that a part with alternatives has, and rows just longer, which
    are cut though there are many of them; all rows' choices, candidates beyond the list among them."""
    V = batches * 1024 * (4 if dtype == F32 else 8) + more
    if batches > 16:
        T //= 4 if dtype != F32 else 2
    say(f"alternatives T={T} V={V} k={k} {dtype}")
    x = _mixed(T, V, dtype, V + k)
    r = lg.logprobs_forward(x, None, k, 0.9, entropy=k == 20)
    place = torch.arange(V - 1, -1, -1, device=DEV)
    for a in range(0, T, 128):
        l = x[a:a + 128].float() + 0.0  # (-0 + 0 = 0)
        bits = l.view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 20) + place  # larger logits, lower places first
        at = torch.topk(order, k, 1).indices
        d = l.double()
        m = d.max(1, keepdim=True).values
        e = torch.exp(0.9 * (d - m))
        S = e.sum(1, keepdim=True)
        mean = torch.where(e > 0, e * 0.9 * (m - d), 0.0).sum(1, keepdim=True) / S
        own = 0.9 * (m - d.gather(1, at))
        assert torch.equal(r.top_ids[a:a + 128].long(), at), a
        bound = U * (3.5 * own + 3 * S.log() + 2.5 * mean + 4 * CHAIN(V) + 8)
        assert ((r.top[a:a + 128].double() - (-own - S.log())).abs() <= bound).all(), a
        lse = (0.9 * m + S.log())[:, 0]
        assert ((r.lse[a:a + 128].double() - lse).abs() <= U * (4 * lse.abs() + 8 * S[:, 0].log()) + bound[:, 0]).all(), a
