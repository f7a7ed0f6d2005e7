"""A renormalised teacher on the GPU: what is added to all of a row's log
probabilities has no part in loss and gradient, and what has no value stays one.

Tolerances as in the other tests of distillation, in units of U = 2^-24; log q, of
the difference from the row's largest and the log of their sum, is off by its own
size and (k + 16) U, whatever the log probabilities' size.
"""

import numpy as np
import pytest
import torch

from _gpu import DEV, say
from oracle import logits_ref as ref
from paper_2211_17111_amd import logits as lg
from test_gpu_logits import BF16, F16, F32, TINY, U, Bounds, _logits, _near, _np, _two_calls

pytestmark = pytest.mark.gpu

CASES = [(19, 118, 5, F32), (19, 118, 20, F16), (7, 300, 64, BF16), (7, 1000, 100, F32), (5, 2000, 256, F16),
         (3, 5000, 20, BF16), (3, 20011, 64, F32), (2, 70001, 200, BF16), (520, 66000, 8, BF16), (2, 200003, 16, F16)]


@pytest.mark.parametrize("T,V,k,dtype", CASES)
def test_an_offset_of_the_teacher_has_no_part(T, V, k, dtype):
    say(f"teacher's offset T={T} V={V} k={k} {dtype}")
    rng = np.random.default_rng(V + k)
    # multiples of 2^-10 down to -8, to which 8192 is added exactly
    logits = torch.from_numpy((-rng.integers(0, 8193, (T, k)) / 1024).astype(np.float32)).to(DEV)
    ids = torch.from_numpy(np.stack([rng.permutation(V)[:k] for _ in range(T)])).to(DEV)
    ids[0, 0] = -1
    logits[-1, -1] = float("-inf")
    x = _logits(T, V, dtype, V)
    g = torch.randn(T, generator=torch.Generator().manual_seed(V)).to(DEV)
    want = [*_two_calls(g, x, ids, logits, 0.8, True), *lg.distill_step(g, x, ids, logits, 0.8, True)]
    for offset in (1.0, -100.0, 1024.0, -8192.0, 8192.0 - 8):
        for a, b in zip([*_two_calls(g, x, ids, logits + offset, 0.8, True),
                         *lg.distill_step(g, x, ids, logits + offset, 0.8, True)], want):
            assert torch.equal(a, b), offset
    if T > 100:
        return
    host, hids, ht = _np(x), ids.cpu().numpy(), _np(logits + 8184.0)
    b = Bounds(host, 0.8)
    loss, gradient = ref.distill_ref(host, hids, ht, 0.8, True), ref.distill_backward_ref(_np(g), host, hids, ht, 0.8, True)
    bound, marked, size = np.zeros(T), np.zeros((T, V)), np.zeros(T)
    for t in range(T):
        kept, logq = ref.taught(hids[t], ht[t], V, True)
        q, at = np.exp(logq), hids[t][kept]
        off = U * (3 * np.abs(logq) + k + 16)
        lp, _ = ref.distribution(host[t], 0.8)
        bound[t] = (q * ((off + (k + 8) * U) * np.abs(logq - lp[at]) + off
                         + b.logprob(np.broadcast_to(at, (T, len(at))))[t])).sum() + TINY
        slip = q * (off + (k + 8) * U) / (80 * U)  # (in units of what Bounds.gradient allows for)
        np.add.at(marked[t], at, (q + slip) * abs(float(g[t])))
        size[t] = abs(float(g[t]))
    bound += 2 * U * np.abs(loss)
    allowed = b.gradient(marked, size, np.zeros(T), np.zeros(T), gradient, dtype)
    for i in (0, 2):
        _near(want[i], loss, bound, "loss")
        _near(want[i + 1], gradient, allowed, "gradient")


def test_a_teacher_of_far_slots():
    """Slots of the type's lowest number beside others have no part, and among themselves share alike."""
    low = torch.finfo(F32).min
    for V in (50, 3001, 40000):
        x = _logits(2, V, F32, V)
        ids = torch.tensor([[1, 2, 3, 4], [1, 2, 3, 4]], device=DEV)
        teacher = torch.tensor([[-3.0, low, -4.0, low], [low] * 4], device=DEV)
        same = torch.tensor([[-3.0, -float("inf"), -4.0, -float("inf")], [0.0] * 4], device=DEV)
        g = torch.ones(2, device=DEV)
        for a, b in zip([*_two_calls(g, x, ids, teacher, 1.0, True), *lg.distill_step(g, x, ids, teacher)],
                        [*_two_calls(g, x, ids, same, 1.0, True), *lg.distill_step(g, x, ids, same)]):
            assert torch.equal(a, b)


def test_a_teacher_without_a_value():
    """A NaN or +inf among a row's kept slots: its loss and gradient are NaN, other rows' are what they are."""
    for V in (50, 3001, 40000, 150001):
        x = _logits(4, V, F32, V)
        ids = torch.tensor([[1, 2, 3], [1, 2, 3], [1, 2, -1], [1, 2, 3]], device=DEV)
        teacher = torch.log_softmax(_logits(4, 3, F32, 1), 1)
        g = torch.ones(4, device=DEV)
        clean = [*_two_calls(g, x, ids, teacher, 1.0, True), *lg.distill_step(g, x, ids, teacher)]
        teacher[0, 1], teacher[3, 0], teacher[2, 2] = float("nan"), float("inf"), float("nan")
        for a, b in zip([*_two_calls(g, x, ids, teacher, 1.0, True), *lg.distill_step(g, x, ids, teacher)], clean):
            assert torch.isnan(a[[0, 3]]).all() and torch.equal(a[1:3], b[1:3])
