"""Plain 64-bit forms of a feed-forward part of experts, on the CPU, from their definitions, with the bounds that the kernels' arithmetic gives."""
import math

import torch

from lowbit_reference import HALF, TINY, TOP, U, blocks, step8


def dense(rows, dtype=torch.float64):
    return torch.tensor(rows, dtype=dtype)


def rms_norm(x, weight, residual, eps):
    """(s, y) in 64 bits."""
    s = x.double() if residual is None else x.double() + residual.double()
    mean = s.square().mean(1, keepdim=True) + eps
    inv = torch.where(mean > 0, mean.rsqrt(), torch.zeros_like(mean))
    y = s * inv
    y = torch.where(torch.isfinite(mean), y, torch.full_like(y, math.nan))
    return s, y if weight is None else y * weight.double()


def swiglu(x):
    """(y, relative error of fp32, absolute error): exp2 of a product with log2(e), rounded twice (2 |g| U) and to 2 units, six more roundings;
    exp(g) below 2^-126 counts as 0."""
    g, u = x.double().chunk(2, 1)
    y = g * torch.sigmoid(g) * u
    return y, (2 * g.abs() + 12) * U, (g * u).abs() * 2.0 ** -126


def check_blocks(values, scales, y, err, fmt):
    """8-bit values and scales (rows_per_scale 1) against y in 64 bits, which the kernel has in fp32 within err (absolute)."""
    rows, cols = y.shape
    v, s = values.cpu().float().double(), scales.cpu().double()
    assert s.shape == (-(-cols // 128), rows)
    for _, bj, r, c in blocks(rows, cols, rows):
        part, off = y[r, c], err[r, c]
        good = torch.isfinite(part).all(1)
        assert torch.isnan(s[bj][~good]).all() and torch.isnan(v[r, c][~good]).all()
        part, off, got, scale = part[good], off[good], v[r, c][good], s[bj][good]
        most = part.abs().amax(1)
        want = (most / TOP[fmt]).clamp(min=TINY)
        # the largest is off by no more than the largest error, the scale by one rounding more
        dscale = off.amax(1) / TOP[fmt] + 2 * U * want
        assert ((scale - want).abs() <= dscale).all()
        q = part / want[:, None]
        # the quotient: its value's error, its scale's, one rounding of fp32; then the nearest 8-bit value
        dq = off / want[:, None] + q.abs() * ((dscale / want)[:, None] + 2 * U)
        near = (q.abs() + dq).clamp(max=TOP[fmt])
        assert ((got - q).abs() <= step8(near, fmt) / 2 + dq * 1.01).all()


def route(logits, top_k, score="softmax", bias=None, groups=1, top_groups=1, group_top=2, renormalize=True, scale=1.0):
    """chosen, weights, starts, pairs, places, and the largest distance of a chosen logit from the row's or the choice's largest (for the bound)."""
    x = logits.double()
    tokens, experts = x.shape
    b = torch.zeros(experts, dtype=torch.float64) if bias is None else bias.double()
    compare_logits = bias is None and (groups == 1 or group_top == 1)
    chosen, weights, far = [], [], 0.0
    for t in range(tokens):
        row = x[t]
        if bool(torch.isnan(row).any() | torch.isnan(b).any() | (b == math.inf).any()) or (score == "softmax" and bool((row == math.inf).any())):
            chosen.append(list(range(top_k)))
            weights.append([math.nan] * top_k)
            continue
        most = float(row.max())
        if score == "softmax":
            p = (row - most).exp() if most > -math.inf else torch.zeros(experts, dtype=torch.float64)
            p = p / p.sum() if most > -math.inf else p
        else:
            p = 1.0 / (1.0 + (-row).exp())
        key = row if compare_logits else p + b
        key = torch.where(row == -math.inf, torch.full_like(key, -math.inf), key).tolist()
        key = [k + 0.0 for k in key]
        each = experts // groups
        allowed = range(groups)
        if groups > 1:
            level = []
            for g in range(groups):
                best = sorted(key[g * each:(g + 1) * each], reverse=True)[:group_top]
                if len(best) == 2 and best[1] == -math.inf:
                    best = best[:1]
                level.append(sum(best))
            allowed = sorted(range(groups), key=lambda g: (-level[g], g))[:top_groups]
        can = [e for g in allowed for e in range(g * each, (g + 1) * each) if key[e] > -math.inf]
        picks = sorted(can, key=lambda e: (-key[e], e))[:top_k]
        z = [float(row[e]) for e in picks]
        if renormalize and picks:
            # relative to the largest: sigmoid(z) = e^z / (1 + e^z)
            hi = max(z)
            if score == "softmax":
                w = [math.exp(v - hi) for v in z]
            else:
                w = [math.exp(min(v, 0.0) - min(hi, 0.0)) * (1 + math.exp(-abs(hi))) / (1 + math.exp(-abs(v))) for v in z]
            w = [v / math.fsum(w) for v in w]
            far = max(far, hi - min(z))
        else:
            w = [float(p[e]) for e in picks]
            far = max([far] + ([most - v for v in z] if score == "softmax" else []))
        chosen.append(picks + [-1] * (top_k - len(picks)))
        weights.append([scale * v for v in w] + [0.0] * (top_k - len(picks)))
    chosen = torch.tensor(chosen, dtype=torch.int32).reshape(tokens, top_k)
    return (chosen, torch.tensor(weights, dtype=torch.float64).reshape(tokens, top_k), *places(chosen, experts), far)


def places(chosen, experts):
    """starts, pairs, places of a choice."""
    flat = chosen.flatten().tolist()
    rows = [[] for _ in range(experts)]
    for pair, e in enumerate(flat):
        if e >= 0:
            rows[e].append(pair)
    starts, pairs, where = [0], [-1] * len(flat), [-1] * len(flat)
    for r in rows:
        for i, pair in enumerate(r):
            pairs[starts[-1] + i], where[pair] = pair, starts[-1] + i
        starts.append(starts[-1] + len(r))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return i32(starts), i32(pairs), i32(where).reshape(chosen.shape)


def weight_bound(want, far, experts):
    """exp to 2 units of a difference that is rounded once, quotients and sums of up to 64 partial sums of experts / 64 each."""
    return (2 * min(far, 200.0) + 80 + experts / 64) * U * want.abs() + 2.0 ** -125


def expert_sum(y, weights, where, base):
    """(sums, bound): a multiply-add in fp32 a slot, one rounding to y's type."""
    tokens, top_k = where.shape
    out = torch.zeros((tokens, y.shape[1]), dtype=torch.float64) if base is None else base.double().clone()
    size = out.abs()
    for s in range(top_k):
        at = where[:, s].long()
        there = (at >= 0) & (at < y.shape[0])
        term = weights[:, s:s + 1].double() * y[at.clamp(0, max(0, y.shape[0] - 1))].double()
        out += torch.where(there[:, None], term, torch.zeros_like(term))
        size += torch.where(there[:, None], term.abs(), torch.zeros_like(term))
    return out, (top_k + 1) * U * size * 1.01 + HALF[y.dtype] * out.abs() * 1.01 + torch.finfo(y.dtype).smallest_normal * HALF[y.dtype]
