"""Performance cases of an expert model's answers: the whole expert layer for a
few tokens, log probabilities of tokens with entropy and top alternatives, and
distillation from a teacher's top alternatives.

A case is one pass.  ``own`` selects the package's kernels; else the pass is
computed from elementary torch operations in float32, rounded once.

Conventions of the operators:
  - ids (of experts, of tokens) outside their range are dropped: an expert slot
    adds nothing, a given token's log probability is 0 and carries no gradient,
    a teacher's alternative has no part in the loss;
  - a logit of -inf has probability 0; a row of nothing else has no
    distribution: log probabilities -inf, entropy 0, alternatives -1, gradient 0;
  - of equal logits the lower index comes first.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
MAX_BYTES = {"layer": 4.1e9, "logprobs": 2.15e9, "distill": 2.15e9}  # those of the largest listed cases
LOSS_SCALE = {"f32": 1.0, "f16": 1024.0, "bf16": 1.0}  # (float16 training scales its loss, or small gradients vanish)
PADDING = 0.03  # share of positions without a token (-1)


def _layer(name, T, E, k, C, F, dtype):
    case = dict(op="layer", T=T, E=E, k=k, C=C, F=F, dtype=dtype)
    return dict(case, name=name) if name else case


def _logprobs(name, T, V, k, entropy, dtype, train, scale=1.0):
    case = dict(op="logprobs", T=T, V=V, k=k, entropy=entropy, dtype=dtype, train=train, scale=scale)
    return dict(case, name=name) if name else case


def _distill(name, T, V, k, dtype, step, renormalise, scale=1.0):
    case = dict(op="distill", T=T, V=V, k=k, dtype=dtype, step=step, renormalise=renormalise, scale=scale)
    return dict(case, name=name) if name else case


def listed():
    return [
        # The expert layer of one decoding sequence.
        _layer("layer_token", 1, 64, 6, 2048, 1024, "bf16"),
        # Few sequences and sizes that are multiples of nothing.
        _layer("layer_odd", 13, 60, 4, 1001, 357, "f16"),
        # A small model's layer, held in float32.
        _layer("layer_f32", 32, 16, 2, 512, 2048, "f32"),
        # A decoding batch that wakes nearly every expert of a large layer.
        _layer("layer_batch", 64, 128, 8, 4096, 1280, "bf16"),
        # The answer of one sequence: its token's log probability and what else it could have been.
        _logprobs("logprobs_token", 1, 32000, 8, False, "bf16", False),
        # A decoding batch with alternatives and entropy, at a temperature.
        _logprobs("logprobs_batch", 64, 131072, 20, True, "bf16", False, 1.25),
        # Scoring a long prompt.
        _logprobs("logprobs_prompt", 8192, 131072, 0, False, "bf16", False),
        # A policy's step: log probability and entropy forward, then their gradient.
        _logprobs("logprobs_train_odd", 2999, 50021, 0, True, "f16", True),
        # A short training batch, loss and gradient in one call.
        _distill("distill_small", 16, 32000, 16, "f32", True, True),
        # The depth bins of six 40 x 100 maps, taught by a larger net's best bins.
        _distill("distill_bins", 24000, 118, 8, "f32", False, True, 0.5),
        # Loss, then gradient, at odd sizes and a temperature; the teacher's mass not renormalised.
        _distill("distill_odd", 2047, 65537, 50, "f16", False, False, 0.5),
        # A long training batch over a large vocabulary, loss and gradient in one call.
        _distill("distill_train", 4096, 131072, 64, "bf16", True, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    while True:
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        op = rng.choice(["layer", "logprobs", "distill"])
        if op == "layer":
            E = _log(rng, 1, 256)
            k = rng.randint(1, min(E, 10))
            C = rng.choice([80, 512, 1024, 2048, 4096, _log(rng, 8, 8192), _log(rng, 64, 8192)])
            F = rng.choice([64, 320, 1024, 2048, _log(rng, 8, 8192), _log(rng, 64, 4096)])
            case = _layer(None, _log(rng, 1, 64), E, k, C, F, dtype)
        else:
            T = _log(rng, 1, 32768)
            V = rng.choice([118, 32000, 65536, 131072, _log(rng, 2, 262144), _log(rng, 1000, 262144)])
            scale = rng.choice([1.0, 1.0, 0.5, 1.25])
            if op == "logprobs":
                k = rng.choice([0, 0, 1, rng.randint(1, min(V, 64))])
                case = _logprobs(None, T, V, k, rng.random() < 0.5, dtype, rng.random() < 0.5, scale)
            else:
                k = rng.randint(1, min(V, 64))
                case = _distill(None, T, V, k, dtype, rng.random() < 0.5, rng.random() < 0.5, scale)
        if work(case)["bytes"] <= MAX_BYTES[op]:
            return case


def work(case):
    T, s, k = case["T"], SIZE[case["dtype"]], case["k"]
    if case["op"] == "layer":
        C, F, E = case["C"], case["F"], case["E"]
        experts = E * -math.expm1(T * math.log1p(-min(k / E, 1 - 1e-12)))  # expected number of different ones
        return {"bytes": experts * 3 * F * C * s + 2 * T * C * s + 8 * T * k, "flops": 6 * T * k * F * C}
    V = case["V"]
    nbytes, flops = s * T * V, 4 * T * V
    if case["op"] == "logprobs":
        nbytes += 4 * T * (2 + case["entropy"] + 2 * k)
        if case["entropy"]:
            flops += 2 * T * V
        if case["train"]:
            nbytes += s * T * V + 4 * T * (1 + case["entropy"] + k)
            flops += (6 if case["entropy"] else 4) * T * V
        return {"bytes": nbytes, "flops": flops}
    nbytes += s * T * V + T * (8 * k + 8)  # the gradient in full
    return {"bytes": nbytes, "flops": flops + 4 * T * V}


# ------------------------------------------------------------------- inputs

def _vocabulary_logits(g, T, V, dev):
    """A spread of tokens of unequal frequency, one raised well above the rest in most rows."""
    l = torch.randn((T, V), generator=g, device=dev).mul_(1.7)
    l += torch.randn(V, generator=g, device=dev) * 1.5
    favoured = torch.randint(0, V, (T, 1), generator=g, device=dev)
    l.scatter_add_(1, favoured, torch.rand((T, 1), generator=g, device=dev) * 14)
    return l, favoured[:, 0]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    T, k = case["T"], case["k"]
    state = {"case": case}

    def rand(*shape):
        return torch.rand(shape, generator=g, device=dev)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    if case["op"] == "layer":
        E, C, F = case["E"], case["C"], case["F"]
        state["x"] = normal(T, C).to(dt)
        ids = rand(T, E).topk(k, dim=1).indices
        state["ids"] = torch.where(rand(T, k) < 0.01, -1, ids).to(torch.int32)
        state["weights"] = torch.softmax(normal(T, k), dim=1)
        up, down = torch.empty((E, 2 * F, C), dtype=dt, device=dev), torch.empty((E, C, F), dtype=dt, device=dev)
        for e in range(E):
            up[e] = normal(2 * F, C) * C ** -0.5
            down[e] = normal(C, F) * F ** -0.5
        state["up"], state["down"] = up, down
        return state
    V = case["V"]
    l, favoured = _vocabulary_logits(g, T, V, dev)
    if case["op"] == "logprobs":
        # (in a row of twenty only some tokens are allowed)
        barred = rand(T, 1) < 0.05
        if bool(barred.any()):
            some = barred[:, 0].nonzero()[:, 0]
            l[some] = l[some].masked_fill(rand(some.numel(), V) < 0.9, -math.inf)
        state["logits"] = l.to(dt)
        ids = torch.where(rand(T) < 0.6, favoured, torch.randint(0, V, (T,), generator=g, device=dev))
        allowed = torch.isfinite(state["logits"].gather(1, ids[:, None])[:, 0])
        ids = torch.where(allowed, ids, state["logits"].argmax(1))
        state["ids"] = torch.where(rand(T) < PADDING, -1, ids)
        if case["train"]:
            up = LOSS_SCALE[case["dtype"]]
            state["grad_logprob"] = normal(T) * up
            state["grad_entropy"] = normal(T) * (0.1 * up) if case["entropy"] else None
            state["grad_top"] = normal(T, k) * up if k else None
        return state
    # the teacher agrees with the student in part
    state["logits"] = l.to(dt)
    step = max(1, (1 << 27) // V)
    teacher, ids = [], []
    for a in range(0, T, step):
        t = l[a:a + step] * 0.9 + normal(min(step, T - a), V)
        best = t.mul_(case["scale"]).topk(k, dim=1)
        teacher.append(best.values - torch.logsumexp(t, 1, keepdim=True))
        ids.append(best.indices)
    ids = torch.cat(ids)
    state["teacher"] = torch.cat(teacher)
    state["ids"] = torch.where(rand(T, 1) < PADDING, -1, ids).to(torch.int32)  # (padded positions)
    state["grad_loss"] = (0.5 + rand(T)) * LOSS_SCALE[case["dtype"]]
    return state


# --------------------------------------------------------------- plain forms

def _gated(hidden, F):
    gate = hidden[..., :F]
    return gate / (1 + torch.exp(-gate)) * hidden[..., F:]


def _plain_layer(state):
    case, x, ids, w = state["case"], state["x"].float(), state["ids"], state["weights"]
    E, k, F, up, down = case["E"], case["k"], case["F"], state["up"], state["down"]
    out = torch.zeros_like(x)
    w = torch.where((ids >= 0) & (ids < E), w, 0.0)
    if ids.numel() < E:  # slot by slot
        expert = ids.clamp(0, E - 1).view(-1)
        for s in range(ids.numel()):
            t = s // k
            h = _gated(up.index_select(0, expert[s:s + 1])[0].float() @ x[t], F)
            out[t] += w.view(-1)[s] * (down.index_select(0, expert[s:s + 1])[0].float() @ h)
    else:  # expert by expert, over all tokens
        for e in range(E):
            share = torch.where(ids == e, w, 0.0).sum(1, keepdim=True)
            out += share * (_gated(x @ up[e].float().t(), F) @ down[e].float().t())
    return out.to(state["x"].dtype)


def _statistics(l):
    """Row maximum (0 where there is none), terms e^(l - max) and their sum."""
    m = l.amax(1, keepdim=True)
    m = torch.where(m > -math.inf, m, 0.0)
    e = torch.exp(l - m)
    return m, e, e.sum(1, keepdim=True)


def _at(values, ids, other):
    """values[t, ids[t, j]], `other` where the id is outside."""
    inside = (ids >= 0) & (ids < values.shape[1])
    return torch.where(inside, values.gather(1, torch.where(inside, ids, 0).long()), other)


def _plain_logprobs(state):
    case, k = state["case"], state["case"]["k"]
    l = state["logits"].float() * case["scale"]
    ids = state["ids"][:, None]
    m, e, total = _statistics(l)
    log_total = torch.log(total)
    inside = (ids >= 0) & (ids < case["V"])
    logp = torch.where(total > 0, _at(l, ids, 0.0) - m - log_total, -math.inf)
    out = [torch.where(inside, logp, 0.0)[:, 0], (m + log_total)[:, 0]]
    if case["entropy"]:
        mean = torch.where(e > 0, e * (l - m), 0.0).sum(1, keepdim=True) / total
        entropy = torch.where(total > 0, log_total - mean, 0.0)
        out.append(entropy[:, 0])
    if k:
        best, order = torch.sort(state["logits"].float(), dim=1, descending=True, stable=True)
        best, order = best[:, :k], order[:, :k]
        chosen = best > -math.inf
        out += [torch.where(chosen, best * case["scale"] - m - log_total, -math.inf), torch.where(chosen, order, -1).int()]
    if case["train"]:
        p = torch.where(total > 0, e / total, 0.0)
        g = torch.where(inside & (total > 0), state["grad_logprob"][:, None], 0.0)
        factor = -g
        if k:
            gt = torch.where(chosen, state["grad_top"], 0.0)
            factor = factor - gt.sum(1, keepdim=True)
        grad = p * factor
        if case["entropy"]:
            deviation = torch.where(p > 0, l - m - log_total + entropy, 0.0)
            grad = grad - p * deviation * state["grad_entropy"][:, None]
        grad.scatter_add_(1, torch.where(inside, ids, 0), g)
        if k:
            grad.scatter_add_(1, order, gt)
        out.append((grad * case["scale"]).to(state["logits"].dtype))
    return out


def _plain_distill(state):
    case, ids, t = state["case"], state["ids"], state["teacher"]
    l = state["logits"].float() * case["scale"]
    m, e, total = _statistics(l)
    t = torch.where((ids >= 0) & (ids < case["V"]), t, -math.inf)
    if case["renormalise"]:
        top, terms, mass = _statistics(t)
        t = torch.where(mass > 0, t - top - torch.log(mass), -math.inf)
    q = torch.exp(t)
    logp = _at(l, ids, 0.0) - m - torch.log(total)
    loss = torch.where(q > 0, q * (t - logp), 0.0).sum(1)
    grad = e / total * q.sum(1, keepdim=True)
    grad.scatter_add_(1, torch.where(q > 0, ids, 0).long(), -q)
    grad = grad * (state["grad_loss"] * case["scale"])[:, None]
    return [loss, grad.to(state["logits"].dtype)]


def run(state):
    case = state["case"]
    if not own:
        return {"layer": _plain_layer, "logprobs": _plain_logprobs, "distill": _plain_distill}[case["op"]](state)
    if case["op"] == "layer":
        from paper_2211_17111_amd import rows
        return rows.expert_layer_forward(state["x"], state["up"], state["down"], state["weights"], state["ids"])
    from paper_2211_17111_amd import logits as ops
    l, scale = state["logits"], case["scale"]
    if case["op"] == "logprobs":
        r = ops.logprobs_forward(l, state["ids"], k=case["k"], scale=scale, entropy=case["entropy"])
        out = [r.logprob, r.lse]
        if case["entropy"]:
            out.append(r.entropy)
        if case["k"]:
            out += [r.top, r.top_ids]
        if case["train"]:
            out.append(ops.logprobs_backward(l, r, state["ids"], scale=scale, grad_logprob=state["grad_logprob"],
                                             grad_entropy=state["grad_entropy"], grad_top=state["grad_top"]))
        return out
    renormalise = case["renormalise"]
    if case["step"]:
        return list(ops.distill_step(state["grad_loss"], l, state["ids"], state["teacher"], scale, renormalise))
    loss, stats = ops.distill_forward(l, state["ids"], state["teacher"], scale, renormalise)
    return [loss, ops.distill_backward(state["grad_loss"], l, state["ids"], state["teacher"], stats, scale, renormalise)]


# ---------------------------------------------------------------- definition

def _exact_layer(state):
    case = state["case"]
    E, F = case["E"], case["F"]
    f64 = torch.float64
    x, ids, w = state["x"].to(f64), state["ids"], state["weights"].to(f64)
    out = torch.zeros_like(x)
    for e in range(E):  # by expert: how much each token wants of it
        share = (w * (ids == e)).sum(1)
        tokens = share.nonzero()[:, 0]
        if not tokens.numel():
            continue
        both = x[tokens] @ state["up"][e].to(f64).t()
        h = both[:, :F] * torch.sigmoid(both[:, :F]) * both[:, F:]
        out[tokens] += share[tokens, None] * (h @ state["down"][e].to(f64).t())
    return out


def _exact_logprobs_rows(case, l, ids, g):
    """Outputs of some rows; g: their outgoing gradients."""
    k, V = case["k"], case["V"]
    dev = l.device
    z = l.double() * case["scale"]
    lse = torch.logsumexp(z, 1)
    some_row = (lse > -math.inf)[:, None]  # (a row of barred tokens only has no distribution)
    logp = torch.where(some_row, z - lse[:, None], -math.inf)
    one_hot = (torch.arange(V, device=dev) == ids[:, None])
    out = [torch.where(one_hot, logp, 0.0).sum(1), lse]
    p = torch.exp(logp)
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    if case["entropy"]:
        out.append(entropy)
    if k:
        # (value descending, index ascending) one at a time
        left = l.double().clone()
        top = []
        for _ in range(k):
            best = left.amax(1, keepdim=True)
            at = torch.where(left == best, torch.arange(V, device=dev), V).amin(1, keepdim=True)
            some = best > -math.inf
            top.append((torch.where(some, best * case["scale"] - lse[:, None], -math.inf), torch.where(some, at, -1)))
            left.scatter_(1, at, -math.inf)
        out += [torch.cat([v for v, _ in top], 1), None]
    if case["train"]:
        grad_logprob, grad_entropy, grad_top = g
        upstream = one_hot * some_row * grad_logprob[:, None].double()
        if k:
            for j, (_, at) in enumerate(top):
                some = (at >= 0)[:, 0]
                upstream[some] = upstream[some].scatter_add(1, at[some], grad_top[some, j:j + 1].double())
        if case["entropy"]:
            upstream = upstream - torch.where(p > 0, p * (logp + 1), 0.0) * grad_entropy[:, None].double()
        out.append(case["scale"] * (upstream - p * upstream.sum(1, keepdim=True)))
    return out


def exact(case, seed):
    """The operators' definitions in float64 (integer outputs have none)."""
    state = prepare(case, seed)
    if case["op"] == "layer":
        return _exact_layer(state)
    T, V, k = case["T"], case["V"], case["k"]
    step = max(1, (1 << 26) // V)
    parts = []
    for a in range(0, T, step):
        b = min(a + step, T)
        l, ids = state["logits"][a:b], state["ids"][a:b]
        if case["op"] == "logprobs":
            g = [None if state.get(n) is None else state[n][a:b] for n in ("grad_logprob", "grad_entropy", "grad_top")]
            parts.append(_exact_logprobs_rows(case, l, ids, g))
            continue
        z = l.double() * case["scale"]
        logp = z - torch.logsumexp(z, 1, keepdim=True)
        inside = (ids >= 0) & (ids < V)
        q = torch.exp(state["teacher"][a:b].double()) * inside
        if case["renormalise"]:
            q = q / torch.where(q.sum(1) > 0, q.sum(1), 1.0)[:, None]
        at = torch.where(inside, ids, 0).long()
        target = torch.zeros_like(z).scatter_add_(1, at, q)  # (a teacher's alternatives are different tokens)
        loss = torch.where(target > 0, target * (torch.log(target) - logp), 0.0).sum(1)
        grad = case["scale"] * state["grad_loss"][a:b, None].double() * (q.sum(1, keepdim=True) * torch.exp(logp) - target)
        parts.append([loss, grad])
    return [None if col[0] is None else torch.cat(col) for col in zip(*parts)]
