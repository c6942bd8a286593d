"""The operators around the AlltoAllv, from their definitions, in 64 bits on the CPU (no code of the library)."""
import math

import torch

FINE = torch.float64
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=FINE)
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}     # of a rounding, relative
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}      # half of the smallest step


def scores(p, logits):
    z = logits.to(FINE).clamp(max=torch.finfo(torch.float32).max)
    there = z > -math.inf
    if p.scoring == "sigmoid":
        s = 1 / (1 + torch.exp(-z))
    else:
        top = torch.where(there, z, -math.inf).amax(dim=1, keepdim=True)
        e = torch.where(there, torch.exp(z - top), 0.0)
        s = e / e.sum(dim=1, keepdim=True)
    return z, torch.where(there, s, 0.0), there


def route(p, logits, bias):
    """Expert by expert in plain Python: the best that is left, the first among equals."""
    z, s, there = scores(p, logits)
    T, E = z.shape
    b = torch.zeros(E, dtype=FINE) if bias is None else bias.to(FINE).clamp(max=torch.finfo(torch.float32).max)
    per = E // p.n_group
    idx = torch.full((T, p.topk), -1, dtype=torch.int32)
    w = torch.zeros(T, p.topk, dtype=FINE)
    for t in range(T):
        can = [bool(there[t, e]) and float(b[e]) > -math.inf for e in range(E)]
        biased = (s[t] + b).tolist()
        key = z[t].tolist() if bias is None else biased
        by = key if p.group_top == 1 else biased
        groups = []
        for g in range(p.n_group):
            best = sorted((by[e] for e in range(g * per, (g + 1) * per) if can[e]), reverse=True)[:p.group_top]
            groups.append(sum(best) if best else -math.inf)
        use = sorted(range(p.n_group), key=lambda g: (-groups[g], g))[:p.topk_group]
        left = [e for g in use for e in range(g * per, (g + 1) * per) if can[e]]
        left.sort(key=lambda e: (-key[e], e))
        for r, e in enumerate(left[:p.topk]):
            idx[t, r] = e
            w[t, r] = s[t, e]
    if p.renormalise:                                # from the scores' logarithms: quotients of scores that 64 bits do not hold
        log = torch.where(z >= 0, -torch.log1p(torch.exp(-z)), z - torch.log1p(torch.exp(z))) if p.scoring == "sigmoid" else z
        log = torch.where(idx >= 0, log.gather(1, idx.long().clamp(min=0)), -math.inf)
        w = torch.nan_to_num(torch.softmax(log, dim=1), nan=0.0)
    return idx, w * p.scale


def weights_of(p, z, idx):
    """The weights of a choice as a function of logits in 64 bits (for differences)."""
    top = torch.where(z > -math.inf, z, -1e300).amax(dim=1, keepdim=True)
    s = 1 / (1 + torch.exp(-z)) if p.scoring == "sigmoid" else torch.exp(z - top) / torch.exp(z - top).sum(dim=1, keepdim=True)
    at = idx.long()
    here = (at >= 0) & (at < z.shape[1])
    here &= z.gather(1, at.clamp(0, z.shape[1] - 1)) > -math.inf
    w = torch.where(here, s.gather(1, at.clamp(0, z.shape[1] - 1)), 0.0)
    if p.renormalise:
        w = w / w.sum(dim=1, keepdim=True).clamp(min=1e-300)
    return w * p.scale


def route_backward(p, logits, idx, grad):
    """(gradient, what its terms add up to without their signs) by the chain rule, slot by slot."""
    z, s, there = scores(p, logits)
    T, E = z.shape
    out, size = torch.zeros(T, E, dtype=FINE), torch.zeros(T, E, dtype=FINE)
    for t in range(T):
        slots = [(k, int(idx[t, k])) for k in range(idx.shape[1]) if 0 <= int(idx[t, k]) < E and bool(there[t, int(idx[t, k])])]
        S = sum(float(s[t, e]) for _, e in slots)
        if p.renormalise and S == 0:
            continue
        w = {k: float(s[t, e]) / (S if p.renormalise else 1.0) for k, e in slots}
        g = {k: float(grad[t, k]) * p.scale for k, _ in slots}
        mean = sum(g[k] * w[k] for k, _ in slots)
        absolute = sum(abs(g[k] * w[k]) for k, _ in slots)
        for k, e in slots:
            tail = 1 - float(s[t, e])
            if p.scoring == "sigmoid":
                d = w[k] * tail * (g[k] - (mean if p.renormalise else 0))
                d_size = w[k] * tail * (abs(g[k]) + (absolute if p.renormalise else 0))
            else:
                d, d_size = w[k] * (g[k] - (mean if p.renormalise else 0)), w[k] * (abs(g[k]) + absolute)
            out[t, e] += d
            size[t, e] += d_size
        if p.scoring == "softmax" and not p.renormalise:
            out[t] -= s[t] * mean
            size[t] += s[t] * absolute
    return out, size


def combine(rows, idx, weights, base):
    """(sum, sum of magnitudes)."""
    T, topk = idx.shape
    x = rows.to(FINE).view(T, topk, -1)
    terms = torch.where((idx >= 0).unsqueeze(2), weights.to(FINE).unsqueeze(2) * x, 0.0)
    b = torch.zeros_like(terms[:, 0]) if base is None else base.to(FINE)
    return b + terms.sum(dim=1), b.abs() + terms.abs().sum(dim=1)


def quantize(x):
    """Codes (a byte each) and scale bytes of 32-bit rows: the nearest value of the grid by distance, the even code of two."""
    R, K = x.shape
    v = x.to(FINE).view(R, K // 32, 32)
    most = v.abs().amax(dim=2)
    bad = ~torch.isfinite(v).all(dim=2)
    most = torch.where(bad, 1.0, most)
    e = torch.where(most > 0, torch.frexp(most)[1].long() - 1, -1000)
    e = (e - 2).clamp(-127, 127)
    a = v.abs() / torch.ldexp(torch.ones_like(most), e).unsqueeze(2)
    d = (a.unsqueeze(3) - GRID).abs()
    best = d.amin(dim=3, keepdim=True)
    near = d == best
    first = near.to(torch.int8).argmax(dim=3)
    both = near.sum(dim=3) == 2                       # a tie is between neighbours: the even one of the two
    code = torch.where(both & (first % 2 == 1), first + 1, first)
    code = code + 8 * torch.signbit(v).long()
    code = torch.where(bad.unsqueeze(2), 0, code)
    return code.view(R, K).to(torch.uint8), torch.where(bad, 255, e + 127).to(torch.uint8)


def pack_codes(code):
    return (code[..., 0::2] + 16 * code[..., 1::2]).contiguous()


def decode(codes, scales):
    """Values in 64 bits; NaN under a scale of 255."""
    code = torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2).long()
    v = GRID[code % 8] * (1 - 2 * (code // 8)).to(FINE)
    s = torch.ldexp(torch.ones(scales.shape, dtype=FINE), scales.long() - 127)
    s = torch.where(scales == 255, math.nan, s)
    return v * s.repeat_interleave(32, dim=-1)


def product(x, w, off, cap):
    """(rows times their experts' matrices, the same of magnitudes); zeros elsewhere."""
    out, size = torch.zeros(cap, w.shape[1], dtype=FINE), torch.zeros(cap, w.shape[1], dtype=FINE)
    for e in range(w.shape[0]):
        a, b = int(off[e]), int(off[e + 1])
        if b > a:
            out[a:b] = x[a:b] @ w[e].T
            size[a:b] = x[a:b].abs() @ w[e].abs().T
    return out, size
