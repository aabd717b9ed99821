"""Plain 64-bit forms of the token operators (router, grouped products, expert
layers, low-rank adapters), with elementwise bounds of what the library's
roundings may add.  Torch on the CPU, loops over rows and groups; no code shared
with the library.

Bounds: a product's fp32 accumulation of n terms is off by at most
n * 2^-24 * sum |terms| to first order, taken with 16 more roundings for the
bias, the activation's evaluation and the combination (the exponential is off
by 2^-22 relative at the arguments that matter); storing a value of type T
rounds by at most u(T) relative, half a step.  The activations are Lipschitz
with a constant below 1.13.
"""
from __future__ import annotations

import math

import torch

EPS32 = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
#: half a step of the subnormals, where the relative bound ends
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
NONE, RELU, RELU6, SILU, GELU = range(5)
LIPSCHITZ = {NONE: 1.0, RELU: 1.0, RELU6: 1.0, SILU: 1.13, GELU: 1.13}
MORE = 16  # roundings besides the accumulation


def act(v, kind):
    if kind == RELU:
        return v.clamp(min=0)
    if kind == RELU6:
        return v.clamp(min=0, max=6)
    if kind == SILU:
        return v * torch.sigmoid(v)
    if kind == GELU:
        return 0.5 * v * torch.erfc(-v / math.sqrt(2))
    return v


def stored(y, err, dtype):
    """The bound of a value with error `err` once it is stored as dtype."""
    return err + UNIT[dtype] * (y.abs() + err) + TINY[dtype]


def linear(x, w, b, kind=NONE):
    """act(x w^T + b) in 64 bits and the bound of its fp32 evaluation; x may
    come as (value, error)."""
    x, ex = x if isinstance(x, tuple) else (x.double(), None)
    w = w.double()
    s = x @ w.t()
    size = x.abs() @ w.abs().t()
    if b is not None:
        s = s + b.double()
        size = size + b.double().abs()
    err = (x.shape[1] + MORE) * EPS32 * size
    if ex is not None:
        err = err + ex @ w.abs().t()
    return act(s, kind), LIPSCHITZ[kind] * err


def route(logits, top_k, bias=None, mask=None, sigmoid=False, renormalize=False, scale=1.0):
    """expert, weight, rows, starts as Python lists and tensors."""
    tokens, experts = logits.shape
    l32 = logits.float()
    key32 = l32 if bias is None else l32 + bias.float()
    expert = torch.full((tokens, top_k), -1, dtype=torch.int32)
    weight = torch.zeros((tokens, top_k), dtype=torch.float64)
    for t in range(tokens):
        if mask is not None and not int(mask[t]):
            continue
        keys, l = key32[t].tolist(), l32[t].tolist()
        live = [e for e in range(experts) if keys[e] > -math.inf]
        chosen = sorted(live, key=lambda e: (-keys[e], e))[:top_k]
        if not chosen:
            continue
        if sigmoid:
            # the sigmoids' logarithms, which do not underflow
            logs = [v - math.log1p(math.exp(v)) if v < 0 else -math.log1p(math.exp(-v)) for v in (l[e] for e in chosen)]
            top = max(logs) if renormalize else 0.0
            s = [math.exp(v - top) for v in logs]
            total = sum(s) if renormalize else 1.0
            w = [v / total for v in s]
        else:
            of = chosen if renormalize else live
            top = max(l[e] for e in of)
            ex = {e: 1.0 if l[e] == top else math.exp(l[e] - top) for e in set(of) | set(chosen)}
            total = sum(ex[e] for e in of)
            w = [ex[e] / total for e in chosen]
        for j, e in enumerate(chosen):
            expert[t, j] = e
            weight[t, j] = scale * w[j]
    rows, starts = [], [0]
    flat = expert.reshape(-1).tolist()
    by = [[] for _ in range(experts)]
    for a, e in enumerate(flat):
        if e >= 0:
            by[e].append(a)
    for g in by:
        rows += g
        starts.append(len(rows))
    rows += [-1] * (len(flat) - len(rows))
    return expert, weight, torch.tensor(rows, dtype=torch.int32), torch.tensor(starts, dtype=torch.int32)


def route_of(logits, expert, mask=None, sigmoid=False, renormalize=False, scale=1.0):
    """weight, rows and starts of a choice that is given (softmax over the experts whose
    logits are neither NaN nor -inf)."""
    l = logits.double()
    there = expert >= 0
    chosen = l.gather(1, expert.long().clamp(min=0)).masked_fill(~there, -math.inf)
    of = chosen if renormalize else l.masked_fill(~(l > -math.inf), -math.inf)
    score = torch.nn.functional.logsigmoid if sigmoid else (lambda v: v)
    logs = score(chosen)
    if sigmoid and not renormalize:
        total = torch.zeros_like(logs[:, :1])
    else:
        total = torch.logsumexp(score(of), 1, keepdim=True)
    weight = (scale * torch.exp(logs - total)).masked_fill(~there, 0.0)
    flat = torch.where(there, expert.long(), logits.shape[1]).reshape(-1)
    rows = torch.sort(flat, stable=True).indices
    starts = (flat[None] < torch.arange(logits.shape[1] + 1)[:, None]).sum(1)
    rows = torch.where(torch.arange(flat.numel()) < starts[-1], rows, -1)
    return weight, rows.to(torch.int32), starts.to(torch.int32)


def grouped(x, y, w, b, starts, src=None, src_div=1, dst=None, kind=NONE):
    """(y in 64 bits with the rows that no position names as they were, bound)."""
    out, bound = y.double().clone(), torch.zeros_like(y, dtype=torch.float64)
    n = len(src) if src is not None else len(dst) if dst is not None else min(x.shape[0], y.shape[0])
    cut = [max(0, min(int(v), n)) for v in starts]
    for g in range(w.shape[0]):
        for p in range(cut[g], cut[g + 1]):
            s = int(src[p]) if src is not None else p
            d = int(dst[p]) if dst is not None else p
            if s < 0 or s // src_div >= x.shape[0] or not 0 <= d < y.shape[0]:
                continue
            v, e = linear(x[s // src_div][None], w[g], None if b is None else b[g], kind)
            out[d], bound[d] = v[0], stored(v, e, y.dtype)[0]
    return out, bound


def halved(y, err, dtype):
    """The same for a value stored as two of dtype, the second what the first left."""
    return err + UNIT[dtype] ** 2 * (y.abs() + err) + TINY[dtype]


def experts(x, weights, expert, weight, residual=False, few=False):
    """weights: dict w_expand, w_gate, w_project, b_* (None: absent), act.  few: a call
    of so few tokens that the hidden rows keep two values of a 16-bit type."""
    tokens = x.shape[0]
    c_out = weights["w_project"].shape[1]
    y = torch.zeros((tokens, c_out), dtype=torch.float64)
    err, size = torch.zeros_like(y), torch.zeros_like(y)

    def of(name, e):
        return None if weights.get(name) is None else weights[name][e]

    for t in range(tokens):
        for j in range(expert.shape[1]):
            e = int(expert[t, j])
            if not 0 <= e < weights["w_expand"].shape[0]:
                continue
            row = x[t][None]
            if weights.get("w_gate") is not None:
                v, ev = linear(row, of("w_expand", e), of("b_expand", e))
                g, eg = linear(row, of("w_gate", e), of("b_gate", e), weights["act"])
                h, eh = v * g, v.abs() * eg + g.abs() * ev + eg * ev + MORE * EPS32 * (v * g).abs()
            else:
                h, eh = linear(row, of("w_expand", e), of("b_expand", e), weights["act"])
            keep = halved if few and x.dtype != torch.float32 else stored
            o, eo = linear((h, keep(h, eh, x.dtype)), of("w_project", e), of("b_project", e))
            k = float(weight[t, j])
            y[t] += k * o[0]
            err[t] += abs(k) * eo[0]
            size[t] += abs(k) * (o[0].abs() + eo[0])
    if residual:
        y += x.double()
        size += x.double().abs()
    err += (expert.shape[1] + 1) * EPS32 * size
    return y, stored(y, err, x.dtype)


def adapted(x, w, b, down, up, ids, scales=None, ranks=None, kind=NONE, halves=False):
    """halves: the first half of an adapter keeps two values of a 16-bit type, so that
    twice as many terms are added to the projection's sum."""
    rows, n = x.shape[0], down.shape[0]
    y, bound = torch.zeros((rows, w.shape[0]), dtype=torch.float64), torch.zeros((rows, w.shape[0]), dtype=torch.float64)
    keep = halved if halves and x.dtype != torch.float32 else stored
    for i in sorted(set(ids.tolist())):
        at = torch.nonzero(ids == i).flatten()
        s, e = linear(x[at], w, b)
        if 0 <= i < n:
            rank = down.shape[1] if ranks is None else max(0, min(int(ranks[i]), down.shape[1]))
            k = 1.0 if scales is None else float(scales[i])
            v, ev = linear(x[at], down[i, :rank], None)
            v, ev = k * v, abs(k) * ev
            a, ea = linear((v, keep(v, ev, x.dtype)), up[i, :, :rank], None)
            more = MORE + (2 * rank if halves else 0)
            s, e = s + a, e + ea + more * EPS32 * (s.abs() + a.abs())
        s, e = act(s, kind), LIPSCHITZ[kind] * e
        y[at], bound[at] = s, stored(s, e, x.dtype)
    return y, bound
