"""Expert layer of a few tokens on the GPU against its float64 oracle.

Tolerances, in units of U = 2^-24: a sum of m products formed in float32 in any
order is off by (m + 2) U of its terms' magnitudes.  The gated product takes 8 U
more.  For a 16-bit type hidden is held as two values of it, whose sum is off by
the square of half a step, and not below float16's smallest number.  Storing
rounds by half a step of the type.
"""

import numpy as np
import pytest
import torch

from _gpu import DEV, say
from oracle import rows_ref as ref
from paper_2211_17111_amd import BevpoolError, rows

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
U = 2.0 ** -24


def _np(t):
    return t.detach().double().cpu().numpy()


def _inputs(T, k, E, C, F, dtype, seed=0, kind="even", wdt=F32):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, by=1.0):
        return (torch.randn(shape, generator=g) * by).to(dtype).to(DEV)

    x, up, down = normal(T, C), normal(E, 2 * F, C, by=C ** -0.5), normal(E, C, F, by=F ** -0.5)
    w = torch.softmax(torch.randn((T, k), generator=g), 1).to(wdt).to(DEV)
    if kind == "even":    # different experts, as a router chooses
        ids = torch.rand((T, E), generator=g).topk(k, 1).indices if k <= E else torch.randint(0, E, (T, k), generator=g)
        ids = torch.where(torch.rand((T, k), generator=g) < 0.1, -1, ids)
    elif kind == "one":   # every slot the same expert
        ids = torch.full((T, k), E - 1)
    elif kind == "none":
        ids = torch.full((T, k), E)
    else:                 # any, several times for a token too, and some outside
        ids = torch.randint(-2, E + 2, (T, k), generator=g)
    return x, up, down, w, ids.to(torch.int32).to(DEV)


def _check(x, up, down, w, ids, label=""):
    T, k = w.shape
    C, F = down.shape[1:]
    out = rows.expert_layer_forward(x, up, down, w, ids)
    assert out.dtype == x.dtype and out.shape == x.shape
    want, size, slip, reach = ref.expert_layer_ref(_np(x), _np(up), _np(down), _np(w), ids.cpu().numpy())
    f = torch.finfo(x.dtype)
    split = U if x.dtype == F32 else (f.eps / 2) ** 2
    bound = (C + 4) * U * slip + (split + (F + k + 16) * U) * size + (2.0 ** -25 if x.dtype == F16 else 2.0 ** -126) * reach
    bound = bound * (1 + 1e-4) + np.abs(want) * f.eps / 2 + f.smallest_normal * f.eps / 2
    err = np.abs(_np(out) - want)
    bad = ~(err <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{label}: {int(bad.sum())} of {err.size} out of tolerance, first at {i}: got {_np(out)[i]}, "
                             f"want {want[i]}, bound {bound[i]}")
    return out


SHAPES = [(1, 1, 1, 1, 1), (1, 6, 64, 256, 128), (2, 2, 4, 7, 5), (5, 3, 3, 33, 17), (1, 8, 8, 80, 320), (13, 4, 60, 101, 57),
          (16, 2, 16, 80, 64), (17, 1, 2, 64, 40), (32, 2, 16, 128, 96), (64, 8, 128, 64, 32), (64, 2, 3, 96, 48),
          (3, 10, 16, 1000, 24), (70, 5, 7, 40, 200), (9, 2, 200, 16, 8), (4, 4, 4, 520, 264), (1, 64, 100, 48, 30)]


@pytest.mark.parametrize("kind", ["even", "one", "none", "any"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,C,F", SHAPES)
def test_expert_layer(T, k, E, C, F, dtype, kind):
    say(f"expert layer T={T} k={k} E={E} C={C} F={F} {dtype} {kind}")
    for wdt in {F32, dtype}:
        out = _check(*_inputs(T, k, E, C, F, dtype, T + C, kind, wdt), kind)
        if kind == "none":
            assert not out.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,C,F", [(512, 2, 30, 64, 48), (1024, 1, 5, 24, 40), (1, 1024, 64, 32, 16), (128, 8, 1000, 16, 24),
                                       (16, 64, 1024, 8, 8), (2, 2, 4, 8192, 64), (2, 2, 4, 64, 8192), (1, 1, 1, 65536, 16)])
def test_borders(T, k, E, C, F, dtype):
    """The most slots, experts and columns."""
    say(f"expert layer T={T} k={k} E={E} C={C} F={F} {dtype}")
    for kind in ("even", "any", "one") if T * k * C * F < 1 << 22 else ("even",):
        _check(*_inputs(T, k, E, C, F, dtype, 3, kind), kind)


def test_large_layer_against_the_device():
    """A decoding batch's size, in float64 on the device."""
    T, k, E, C, F = 64, 8, 64, 2048, 1024
    for dtype in (BF16, F16):
        say(f"large layer {dtype}")
        x, up, down, w, ids = _inputs(T, k, E, C, F, dtype)
        out = rows.expert_layer_forward(x, up, down, w, ids)
        want = torch.zeros((T, C), dtype=torch.float64, device=DEV)
        size = torch.zeros_like(want)
        for e in range(E):
            share = (w * (ids == e)).sum(1)
            t = share.nonzero()[:, 0]
            both = x[t].double() @ up[e].double().t().contiguous()
            h = both[:, :F] * torch.sigmoid(both[:, :F]) * both[:, F:]
            want[t] += share[t, None].double() * (h @ down[e].double().t().contiguous())
            size[t] += share[t, None].double() * (h.abs() @ down[e].double().abs().t().contiguous())
        # (errors of gate and value are far below hidden's own here: 40 covers them)
        eps = torch.finfo(dtype).eps / 2
        assert ((out.double() - want).abs() <= want.abs() * eps + size * (eps ** 2 + (C + F + 40) * U) + 1e-7).all()


def test_what_is_not_chosen_is_not_read():
    """NaN in experts without a slot, in tokens without an expert, and in dropped slots' weights reach nothing."""
    for dtype in TYPES:
        x, up, down, w, ids = _inputs(9, 3, 12, 70, 33, dtype, 1)
        ids[ids == 5] = 6
        ids[4] = -1
        clean = rows.expert_layer_forward(x, up, down, w, ids)
        up[5], down[5], x[4] = float("nan"), float("inf"), float("nan")
        w[ids < 0] = float("nan")
        dirty = rows.expert_layer_forward(x, up, down, w, ids)
        assert torch.equal(clean, dirty) and not dirty[4].any()


def test_nan_and_inf_stay_with_their_token():
    for dtype in TYPES:
        x, up, down, w, ids = _inputs(20, 2, 3, 40, 24, dtype, 2)
        ids[7, 0] = 1
        clean = rows.expert_layer_forward(x, up, down, w, ids)
        x[7, 3] = float("nan")
        out = rows.expert_layer_forward(x, up, down, w, ids)
        assert torch.isnan(out[7]).all()
        rest = [t for t in range(20) if t != 7]
        assert torch.equal(out[rest], clean[rest])


def test_the_same_call_twice_gives_the_same_bits():
    """However an expert's slots arrive in their list."""
    for T, k, E in ((64, 8, 12), (512, 2, 3), (3, 4, 8)):
        args = _inputs(T, k, E, 96, 320, BF16, 7, "any")
        want = rows.expert_layer_forward(*args)
        for _ in range(4):
            assert torch.equal(rows.expert_layer_forward(*args), want)


def test_large_gates():
    """silu at both ends: a gate far below zero gives 0, one far above is itself."""
    for dtype in TYPES:
        x = torch.ones((2, 8), dtype=dtype, device=DEV)
        x[1] = -1
        up = torch.ones((1, 2, 8), dtype=dtype, device=DEV)
        up[0, 0] = 30  # gates of 240 and -240, values of 8 and -8
        down = torch.ones((1, 8, 1), dtype=dtype, device=DEV)
        out = rows.expert_layer_forward(x, up, down, torch.ones((2, 1), device=DEV),
                                        torch.zeros((2, 1), dtype=torch.int32, device=DEV))
        assert (out[0] == 1920).all() and (out[1].float().abs() < 1e-30).all()


def test_strided_tokens_and_unaligned_weights():
    for dtype in TYPES:
        for C in (64, 75):
            x, up, down, w, ids = _inputs(6, 2, 5, C, 40, dtype, 4)
            want = rows.expert_layer_forward(x, up, down, w, ids)
            wide = torch.zeros((6, 2 * C + 3), dtype=dtype, device=DEV)
            wide[:, 5:5 + C] = x
            assert torch.equal(rows.expert_layer_forward(wide[:, 5:5 + C], up, down, w, ids), want)
            off = [torch.zeros(t.numel() + 1, dtype=dtype, device=DEV)[1:].view(t.shape).copy_(t) for t in (up, down)]
            assert torch.equal(rows.expert_layer_forward(x, *off, w, ids), want)
            one = rows.expert_layer_forward(x[:1].expand(6, C), up, down, w, ids)
            assert torch.equal(one, rows.expert_layer_forward(x[:1].repeat(6, 1), up, down, w, ids))


def test_places_past_32_bits():
    """An expert's rows more than 2^32 elements into the weights."""
    E, C, F = 5, 32768, 16384  # up: 5 x 2^30 elements, 10.7 GB
    up = torch.zeros((E, 2 * F, C), dtype=BF16, device=DEV)
    down = torch.zeros((E, C, F), dtype=BF16, device=DEV)
    x = torch.zeros((1, C), dtype=BF16, device=DEV)
    x[0, -1] = 1
    up[4, F - 1, -1], up[4, 2 * F - 1, -1] = 2, 3
    down[4, -1, -1], down[4, 5, F - 1] = 0.5, -4
    out = rows.expert_layer_forward(x, up, down, torch.ones((1, 2), device=DEV),
                                    torch.tensor([[4, 0]], dtype=torch.int32, device=DEV))
    h = 6 / (1 + np.exp(-2))
    assert abs(float(out[0, -1]) - h / 2) < 0.02 and abs(float(out[0, 5]) + 4 * h) < 0.1
    out[0, -1] = out[0, 5] = 0
    assert not out.any()


def test_no_tokens_other_stream_and_graph():
    x, up, down, w, ids = _inputs(8, 4, 16, 96, 64, BF16, 5)
    none = rows.expert_layer_forward(x[:0], up, down, w[:0], ids[:0])
    assert none.shape == (0, 96)
    want = rows.expert_layer_forward(x, up, down, w, ids)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = rows.expert_layer_forward(x, up, down, w, ids, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = rows.expert_layer_forward(x, up, down, w, ids)
        graphs.append((graph, out))
    for i in range(3):
        y, _, _, v, j = _inputs(8, 4, 16, 96, 64, BF16, 20 + i, "any")
        x.copy_(y), w.copy_(v), ids.copy_(j)
        want = rows.expert_layer_forward(x, up, down, w, ids)
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert torch.equal(out, want)


def test_refusals():
    x, up, down, w, ids = _inputs(4, 2, 3, 16, 8, BF16)
    bad = [(x.float(), up, down, w, ids), (x, up.float(), down, w, ids), (x, up[:, :15], down, w, ids), (x, up[:2], down, w, ids),
           (x, up.transpose(1, 2), down, w, ids), (x, up, down[:, :8], w, ids), (x, up, down, w[:3], ids[:3]),
           (x, up, down, w.to(F16), ids), (x, up, down, w, ids.long()), (x, up, down, w, ids[:, :1]), (x.t(), up, down, w, ids),
           (x, up, down, w.cpu(), ids)]
    for args in bad:
        with pytest.raises(ValueError):
            rows.expert_layer_forward(*args)
    many = _inputs(513, 2, 3, 16, 8, BF16)
    with pytest.raises(BevpoolError):
        rows.expert_layer_forward(*many)
