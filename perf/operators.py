"""The operators around one expert-parallel AlltoAllv that a mixture-of-experts layer needs next to the transport, and what
they are measured on.

* ``route``            -- router logits to experts and weights (what ``demand_from_routing`` and ``pack`` take)
* ``route_backward``   -- gradient of the weights with respect to the logits
* ``combine``          -- the returned rows (what ``unpack_tokens`` writes) summed with their weights
* ``combine_backward`` -- gradients of the rows and of the weights
* ``wire``             -- rows to 4-bit codes with a scale per 32 values, as ``pack`` sends them, and back to values
* ``product``          -- expert-major rows (what ``unpack`` writes) times the experts' matrices, both in that format
* ``experts``          -- a rank's experts as a layer runs them: up and gate, activation and rounding, down

Every operator has a plain form of elementary tensor operations; the framework's calls take the same state.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
BLOCK = 32                                   # values that share a scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)     # what three bits of a code stand for; the fourth is the sign


# ---- cases --------------------------------------------------------------------------------------------------------------

def listed():
    grouped = dict(scoring="sigmoid", bias=True, n_group=8, topk_group=4, group_top=2, renormalise=True, scale=2.5, masked=False)
    return [
        # a decode step's routing, on the critical path of every layer: sigmoid scores, balance bias, 4 of 8 groups
        dict(name="route_decode", kind="route", tokens=128, experts=256, topk=8, dtype="fp32", **grouped),
        # the same for a long prefill
        dict(name="route_prefill", kind="route", tokens=16384, experts=256, topk=8, dtype="fp32", **grouped),
        # training step: softmax scores as they are, every logit gets a gradient
        dict(name="route_backward_train", kind="route_backward", tokens=16384, experts=128, topk=8, dtype="bf16", scoring="softmax",
             bias=False, n_group=1, topk_group=1, group_top=1, renormalise=False, scale=1.0, masked=False),
        # a ragged micro-batch with padding tokens and experts that are switched off
        dict(name="route_backward_ragged", kind="route_backward", tokens=1531, experts=192, topk=6, dtype="fp32", scoring="sigmoid",
             bias=True, n_group=1, topk_group=1, group_top=1, renormalise=True, scale=1.0, masked=True),
        # the end of a decode step's layer, with a shared expert's output underneath
        dict(name="combine_decode", kind="combine", tokens=128, topk=8, hidden=7168, dtype="bf16", base=True, dropped=0.0),
        # the end of a prefill's layer
        dict(name="combine_prefill", kind="combine", tokens=16384, topk=8, hidden=7168, dtype="bf16", base=False, dropped=0.0),
        # training: a micro-batch, and a ragged one with dropped copies
        dict(name="combine_backward_train", kind="combine_backward", tokens=8192, topk=8, hidden=4096, dtype="bf16", dropped=0.0),
        dict(name="combine_backward_ragged", kind="combine_backward", tokens=1531, topk=6, hidden=2048, dtype="bf16", dropped=0.1),
        # rows on their way through a dispatch: a decode step's and a prefill's
        dict(name="wire_decode", kind="wire", rows=128, cols=7168, dtype="bf16"),
        dict(name="wire_prefill", kind="wire", rows=16384, cols=7168, dtype="bf16"),
        # a decode step's rows on a rank with 16 experts: the matrices have to be read, and little else
        dict(name="product_decode", kind="product", experts=16, rows=128, spare=128, cols=7168, outputs=4096, dtype="bf16", skew=0.8),
        # a prefill on a rank with 8 experts
        dict(name="experts_prefill", kind="experts", experts=8, rows=16384, spare=4096, cols=7168, outputs=2048, dtype="bf16", skew=0.8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "route", "route_backward", "combine", "combine_backward", "wire", "product", "product", "experts"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind in ("route", "route_backward"):
        E = rng.choice([8, 16, 60, 64, 96, 128, 160, 192, 256])
        n_group = rng.choice([1, 1, 2, 4, 8]) if E % 8 == 0 else 1
        topk_group = rng.randint(1, n_group)
        topk = min(rng.choice([1, 2, 4, 6, 8]), topk_group * (E // n_group))
        return dict(kind=kind, tokens=_log_int(rng, 1, 16384), experts=E, topk=topk, dtype=dtype, scoring=rng.choice(["softmax", "sigmoid"]),
                    bias=rng.random() < 0.5, n_group=n_group, topk_group=topk_group, group_top=rng.choice([1, 2]),
                    renormalise=topk > 1 and rng.random() < 0.6, scale=rng.choice([1.0, 2.5]),     # (one weight of 1 has no gradient)
                    masked=topk_group * (E // n_group) >= 32 and rng.random() < 0.4)
    if kind in ("combine", "combine_backward"):
        topk, hidden = rng.choice([1, 2, 4, 6, 8]), rng.choice([_log_int(rng, 8, 8192), 1024, 2048, 4096, 7168])
        most = max(2, min(16384, (1 << 30) // (topk * hidden * BYTES[dtype])))
        case = dict(kind=kind, tokens=_log_int(rng, 1, most), topk=topk, hidden=hidden, dtype=dtype, dropped=rng.choice([0.0, 0.1, 0.9]))
        return dict(case, base=rng.random() < 0.5) if kind == "combine" else case
    if kind == "wire":
        cols = 32 * rng.choice([_log_int(rng, 1, 256), 64, 128, 224])
        return dict(kind=kind, rows=_log_int(rng, 1, max(2, min(16384, (1 << 27) // cols))), cols=cols, dtype=dtype)
    E = rng.choice([1, 2, 4, 8, 16, 32])
    cols = 32 * rng.choice([_log_int(rng, 1, 224), 32, 64, 224])
    outputs = rng.choice([_log_int(rng, 8, 4096), 1024, 2048, 4096]) if kind == "product" else 32 * _log_int(rng, 1, 64)
    most = max(2, min(8192, (1 << 37) // (cols * outputs)))
    rows = _log_int(rng, 1, most)
    return dict(kind=kind, experts=E, rows=rows, spare=rng.choice([0, 1, 100]), cols=cols, outputs=outputs,
                dtype=dtype if kind == "product" else "bf16", skew=rng.choice([0.0, 0.8, 1.2]))


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _randn(shape, gen, dtype=torch.float32):
    return torch.randn(shape, device=DEVICE, generator=gen, dtype=dtype)


def _zeros(*shape, dtype=torch.float32):
    return torch.zeros(shape, device=DEVICE, dtype=dtype)


def _logits(case, gen):
    T, E = case["tokens"], case["experts"]
    z = _randn((T, E), gen) * 1.2 + _randn((1, E), gen) * 0.5            # some experts are liked more
    if case["masked"]:                                                  # experts switched off, padding tokens
        z = z.masked_fill(torch.rand(1, E, device=DEVICE, generator=gen) < 0.1, -math.inf)
        z = z.masked_fill(torch.rand(T, 1, device=DEVICE, generator=gen) < 0.05, -math.inf)
    return z.to(DTYPES[case["dtype"]]).contiguous()


def _bias(case, gen):
    """A balance bias as it stands after some steps of +-0.001."""
    return torch.round(_randn((case["experts"],), gen) * 20) / 1000 if case["bias"] else None


def _routing(case, gen):
    T, topk = case["tokens"], case["topk"]
    idx = torch.randint(0, 256, (T, topk), device=DEVICE, generator=gen, dtype=torch.int32)
    idx = torch.where(torch.rand(T, topk, device=DEVICE, generator=gen) < case["dropped"], -1, idx)
    w = torch.rand(T, topk, device=DEVICE, generator=gen) + 0.05
    return idx.contiguous(), (w / w.sum(dim=1, keepdim=True)).contiguous()


def _activations(shape, gen):
    """Normal values; one column in 50 is ten times as large, as hidden states are."""
    x = _randn(shape, gen)
    return x * torch.where(torch.rand(shape[-1], device=DEVICE, generator=gen) < 0.02, 10.0, 1.0)


def _wire_rows(rows, cols):
    """A buffer of rows as they are sent, and its two parts: codes, scales behind them, rows of whole 16 bytes."""
    buf = _zeros(rows, (cols // 2 + cols // BLOCK + 15) // 16 * 16, dtype=torch.uint8)
    return buf, buf[:, :cols // 2], buf[:, cols // 2:cols // 2 + cols // BLOCK]


def _matrices(E, outputs, cols, gen):
    """``E`` experts' matrices, codes ``[E, outputs, cols / 2]`` and scales ``[E, outputs, cols / 32]``."""
    code, scale = _encode(_randn((E * outputs, cols), gen) / math.sqrt(cols))
    return _nibbles(code).view(E, outputs, cols // 2), scale.view(E, outputs, cols // BLOCK)


def _offsets(case, gen):
    """First row of each expert and the end: popularities (1 + rank)^-skew in a random order."""
    E = case["experts"]
    p = (1 + torch.rand(E, device=DEVICE, generator=gen).argsort().to(torch.float32)) ** -case["skew"]
    of = torch.multinomial(p, case["rows"], replacement=True, generator=gen)
    n = torch.bincount(of, minlength=E)
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEVICE), n.cumsum(0)]).to(torch.int32)
    return off, int(n.max())


def prepare(case, seed):
    gen, kind, dt = _gen(seed), case["kind"], DTYPES[case["dtype"]]
    s = {"kind": kind, "case": case}
    if kind in ("route", "route_backward"):
        T, E, topk = case["tokens"], case["experts"], case["topk"]
        s.update(logits=_logits(case, gen), bias=_bias(case, gen), idx=_zeros(T, topk, dtype=torch.int32), weights=_zeros(T, topk))
        if kind == "route_backward":
            s["idx"] = _route_plain(case, s["logits"], s["bias"])[0]
            s.update(grad=_randn((T, topk), gen), out=_zeros(T, E, dtype=dt))
        s["params"] = _params(case)
        return s
    if kind in ("combine", "combine_backward"):
        T, topk, H = case["tokens"], case["topk"], case["hidden"]
        idx, w = _routing(case, gen)
        s.update(idx=idx, weights=w, rows=_randn((T * topk, H), gen, dt))
        if kind == "combine":
            s.update(base=_randn((T, H), gen, dt) if case["base"] else None, out=_zeros(T, H, dtype=dt))
        else:
            s.update(grad=_randn((T, H), gen, dt), grad_rows=_zeros(T * topk, H, dtype=dt), grad_weights=_zeros(T, topk))
        return s
    if kind == "wire":
        R, K = case["rows"], case["cols"]
        buf, codes, scales = _wire_rows(R, K)
        s.update(x=_activations((R, K), gen).to(dt), buf=buf, codes=codes, scales=scales, out=_zeros(R, K, dtype=dt))
        return s
    E, K, F, cap = case["experts"], case["cols"], case["outputs"], case["rows"] + case["spare"]
    off, most = _offsets(case, gen)
    buf, codes, scales = _wire_rows(cap, K)
    code, scale = _encode(_activations((cap, K), gen))
    codes.copy_(_nibbles(code))
    scales.copy_(scale)
    s.update(buf=buf, codes=codes, scales=scales, off=off, most=most, status=_zeros(1, dtype=torch.int32))
    if kind == "product":
        s.update(w=_matrices(E, F, K, gen), out=_zeros(cap, F, dtype=dt))
        return s
    hbuf, hcodes, hscales = _wire_rows(cap, F)                             # (what the activation leaves, in the same format)
    s.update(up=_matrices(E, 2 * F, K, gen), down=_matrices(E, K, F, gen), hidden=_zeros(cap, 2 * F, dtype=dt), hbuf=hbuf, hcodes=hcodes,
             hscales=hscales, out=_zeros(cap, K, dtype=dt))
    return s


def _params(case):
    """The router's settings as a program keeps them; the framework's record is made from them in the call."""
    return {k: case[k] for k in ("experts", "topk", "scoring", "n_group", "topk_group", "group_top", "renormalise", "scale")}


# ---- plain forms --------------------------------------------------------------------------------------------------------

def _scores_plain(scoring, logits):
    """(logits, scores) in 64 bits -- which of two experts is chosen hangs on the last bits of 32 -- and which experts can be
    chosen: those whose logit is a number above -inf."""
    z = logits.double()
    there = z > -math.inf
    z = torch.where(there, z, 0.0)
    if scoring == "sigmoid":
        return z, torch.where(there, 1 / (1 + torch.exp(-z)), 0.0), there
    most = torch.where(there, z, -math.inf).amax(dim=1, keepdim=True)
    e = torch.where(there, torch.exp(z - torch.where(most > -math.inf, most, 0.0)), 0.0)
    total = e.sum(dim=1, keepdim=True)
    return z, e / torch.where(total > 0, total, 1.0), there


def _route_plain(case, logits, bias):
    T, E = logits.shape
    G, topk = case["n_group"], case["topk"]
    z, score, there = _scores_plain(case["scoring"], logits)
    biased = score + (bias.double() if bias is not None else 0.0)
    key = torch.where(there, biased if bias is not None else z, -math.inf)      # (scores rise with logits: no bias, no rounding)
    if G > 1:
        by = key if case["group_top"] == 1 else torch.where(there, biased, -math.inf)
        best = by.view(T, G, E // G).sort(dim=2, descending=True).values[:, :, :case["group_top"]]
        group = torch.where(best[:, :, 0] > -math.inf, torch.where(best > -math.inf, best, 0.0).sum(dim=2), -math.inf)
        order = group.sort(dim=1, descending=True, stable=True).indices[:, :case["topk_group"]]
        inside = torch.zeros(T, G, dtype=torch.bool, device=z.device).scatter_(1, order, True)
        key = torch.where(inside.repeat_interleave(E // G, dim=1), key, -math.inf)
    key, idx = (v[:, :topk] for v in key.sort(dim=1, descending=True, stable=True))
    found = key > -math.inf
    w = torch.where(found, score.gather(1, idx), 0.0)
    if case["renormalise"]:
        total = w.sum(dim=1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
    return torch.where(found, idx, -1).to(torch.int32), (w * case["scale"]).float()


def _route_backward_plain(case, logits, idx, grad):
    z, score, there = _scores_plain(case["scoring"], logits)
    at = idx.long().clamp(min=0)
    here = (idx >= 0) & there.gather(1, at)
    g = torch.where(here, grad.double() * case["scale"], 0.0)
    s = torch.where(here, score.gather(1, at), 0.0)
    if case["renormalise"]:                                                  # w = s / sum: g loses its mean under w
        total = s.sum(dim=1, keepdim=True)
        total = torch.where(total > 0, total, 1.0)
        g = torch.where(here, (g - (g * s).sum(dim=1, keepdim=True) / total) / total, 0.0)
    ds = torch.zeros_like(z).scatter_add_(1, at, g)
    if case["scoring"] == "sigmoid":
        return (ds * score * (1 - score)).to(logits.dtype)
    return (score * (ds - (ds * score).sum(dim=1, keepdim=True))).to(logits.dtype)


def _combine_plain(s):
    T, topk = s["idx"].shape
    rows = s["rows"].view(T, topk, -1).float()
    w = s["weights"].unsqueeze(2)
    out = torch.where(s["idx"].unsqueeze(2) >= 0, w * rows, 0.0).sum(dim=1)
    if s["base"] is not None:
        out = out + s["base"].float()
    return out.to(s["rows"].dtype)


def _combine_backward_plain(s):
    T, topk = s["idx"].shape
    here = s["idx"].unsqueeze(2) >= 0
    grad = s["grad"].float().unsqueeze(1)
    rows = s["rows"].view(T, topk, -1).float()
    grad_rows = torch.where(here, s["weights"].unsqueeze(2) * grad, 0.0)
    grad_weights = torch.where(here, rows * grad, 0.0).sum(dim=2)
    return grad_rows.to(s["rows"].dtype).view(T * topk, -1), grad_weights


def _power(e):
    """2^e, -127 <= e <= 127, from its bits."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _encode(x):
    """Rows in 32 bits to codes (one per byte) and scales (exponent + 127): the scale is the power of two that brings the largest
    of 32 values to [4, 8); values go to the nearest of the grid, ties to the even code, those above 6 to 6."""
    R, K = x.shape
    v = x.view(R, K // BLOCK, BLOCK)
    e = torch.frexp(v.abs().amax(dim=2))[1] - 3
    e = torch.where(v.abs().amax(dim=2) > 0, e, -127).clamp(-127, 127)
    y = v * _power(-e.unsqueeze(2))
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    return (code + 8 * (y < 0).to(torch.uint8)).view(R, K), (e + 127).to(torch.uint8)


def _nibbles(code):
    return (code[..., 0::2] + 16 * code[..., 1::2]).contiguous()


def _decode(codes, scales):
    """Codes and scales to the values they stand for, in 32 bits."""
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    v = grid[torch.stack([codes & 15, codes >> 4], dim=-1).long().view(*codes.shape[:-1], -1)]
    return (v.view(*scales.shape, BLOCK) * _power(scales.int() - 127).unsqueeze(-1)).view(v.shape)


def _product_plain(x, w, off, most, dtype):
    """Rows ``[R, K]`` times the transposed matrices of their experts ``[E, F, K]``, zeros behind the last expert's rows.  Experts' rows side by side, filled up to the longest: one batched product."""
    R, E = x.shape[0], w.shape[0]
    off = off.long()
    at = off[:-1].unsqueeze(1) + torch.arange(most, device=x.device)
    y = torch.bmm(x[at.clamp(max=R - 1)], w.transpose(1, 2))
    row = torch.arange(R, device=x.device)
    expert = torch.searchsorted(off[1:], row, right=True)
    there = expert < E
    expert = expert.clamp(max=E - 1)
    y = y[expert, (row - off[expert]).clamp(0, most - 1)]
    return torch.where(there.unsqueeze(1), y, 0.0).to(dtype)


def _gated(h):
    """silu(first half) * second half."""
    g, u = h.float().chunk(2, dim=1)
    return g / (1 + torch.exp(-g)) * u


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    kind, case = s["kind"], s["case"]
    if kind == "route":
        return _route_plain(case, s["logits"], s["bias"])
    if kind == "route_backward":
        return _route_backward_plain(case, s["logits"], s["idx"], s["grad"])
    if kind == "combine":
        return _combine_plain(s)
    if kind == "combine_backward":
        return _combine_backward_plain(s)
    if kind == "wire":
        code, scale = _encode(s["x"].float())
        s["codes"].copy_(_nibbles(code))
        s["scales"].copy_(scale)
        return _decode(s["codes"], s["scales"]).to(s["x"].dtype)
    x = _decode(s["codes"], s["scales"])
    if kind == "product":
        return _product_plain(x, _decode(*s["w"]), s["off"], s["most"], s["out"].dtype)
    h = _product_plain(x, _decode(*s["up"]), s["off"], s["most"], s["hidden"].dtype)
    code, scale = _encode(_gated(h))
    return _product_plain(_decode(_nibbles(code), scale), _decode(*s["down"]), s["off"], s["most"], s["out"].dtype)


def _run_own(s):
    import paper_2609_34340_b200 as vp
    kind = s["kind"]
    if kind == "route":
        vp.route(vp.RouteParams(**s["params"]), s["logits"], s["bias"], s["idx"], s["weights"])
        return s["idx"], s["weights"]
    if kind == "route_backward":
        vp.route_backward(vp.RouteParams(**s["params"]), s["logits"], s["idx"], s["grad"], s["out"])
        return s["out"]
    if kind == "combine":
        vp.combine(s["rows"], s["idx"], s["weights"], s["base"], s["out"])
        return s["out"]
    if kind == "combine_backward":
        vp.combine_backward(s["grad"], s["rows"], s["idx"], s["weights"], s["grad_rows"], s["grad_weights"])
        return s["grad_rows"], s["grad_weights"]
    if kind == "wire":
        vp.mxfp4_quantize(s["x"], s["codes"], s["scales"])
        vp.mxfp4_dequantize(s["codes"], s["scales"], s["out"])
        return s["out"]
    if kind == "product":
        vp.mxfp4_product(s["codes"], s["scales"], *s["w"], s["off"], s["out"], s["status"])
        return s["out"]
    vp.mxfp4_product(s["codes"], s["scales"], *s["up"], s["off"], s["hidden"], s["status"])
    vp.mxfp4_quantize(s["hidden"], s["hcodes"], s["hscales"], gated=True, n_rows=s["off"][-1:])
    vp.mxfp4_product(s["hcodes"], s["hscales"], *s["down"], s["off"], s["out"], s["status"])
    return s["out"]


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    kind, b = case["kind"], BYTES[case["dtype"]]
    if kind in ("route", "route_backward"):
        T, E, topk = case["tokens"], case["experts"], case["topk"]
        if kind == "route":                                              # logits in, an expert and a weight out
            return {"bytes": T * (E * b + topk * 8), "flops": T * E * (topk + 4)}
        # every gradient out; softmax as it is needs every logit, all else the chosen ones
        every = case["scoring"] == "softmax" and not case["renormalise"]
        return {"bytes": T * (E * b + (E if every else topk) * b + topk * 8), "flops": T * E * 4}
    if kind in ("combine", "combine_backward"):
        T, topk, H = case["tokens"], case["topk"], case["hidden"]
        rows = T * topk * (1 - case["dropped"])
        if kind == "combine":
            return {"bytes": (rows + T * (2 if case["base"] else 1)) * H * b + T * topk * 8, "flops": 2 * rows * H}
        return {"bytes": (rows + T * topk + T) * H * b + T * topk * 12, "flops": 3 * rows * H}
    row = lambda n: n / 2 + n / BLOCK  # noqa: E731
    if kind == "wire":
        R, K = case["rows"], case["cols"]
        return {"bytes": 2 * R * (K * b + row(K)), "flops": 4 * R * K}
    E, R, K, F = min(case["experts"], case["rows"]), case["rows"], case["cols"], case["outputs"]
    if kind == "product":
        return {"bytes": E * F * row(K) + R * (row(K) + F * b), "flops": 2 * R * F * K}
    return {"bytes": E * (2 * F * row(K) + K * row(F)) + R * (row(K) + 2 * 2 * F * b + 2 * row(F) + K * b), "flops": 2 * R * 3 * F * K}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def _exact_route(case, logits, bias):
    """One expert after another: the best that is left, the lowest index among equals."""
    z = torch.nan_to_num(logits.double(), nan=-math.inf, neginf=-math.inf)
    T, E = z.shape
    G, per = case["n_group"], E // case["n_group"]
    if case["scoring"] == "sigmoid":
        score = torch.sigmoid(z)
    else:
        score = torch.nan_to_num(torch.softmax(z, dim=1), nan=0.0)
    value = z if bias is None else torch.where(z == -math.inf, z, score + bias.double())
    open_ = torch.ones(T, G, dtype=torch.bool, device=z.device)
    if G > 1:
        by = torch.where(z == -math.inf, z, score if bias is None else score + bias.double()).view(T, G, per)
        top = by.topk(min(case["group_top"], per), dim=2).values
        of = torch.where(top[:, :, 0] == -math.inf, -math.inf, torch.where(top == -math.inf, 0.0, top).sum(dim=2))
        if bias is None and case["group_top"] == 1:
            of = z.view(T, G, per).amax(dim=2)
        open_ = ~open_
        left = of.clone()
        for _ in range(case["topk_group"]):
            best = (left == left.amax(dim=1, keepdim=True)).to(torch.int8).argmax(dim=1, keepdim=True)
            open_.scatter_(1, best, True)
            left.scatter_(1, best, -math.inf)
            left = torch.where(open_, torch.full_like(left, -math.inf), left)
    value = torch.where(open_.unsqueeze(2).expand(T, G, per).reshape(T, E), value, -math.inf)
    weight = []
    for _ in range(case["topk"]):
        most = value.amax(dim=1, keepdim=True)
        best = (value == most).to(torch.int8).argmax(dim=1, keepdim=True)
        weight.append(torch.where(most > -math.inf, score.gather(1, best), 0.0))
        value = value.scatter(1, best, -math.inf)
    w = torch.cat(weight, dim=1)
    if case["renormalise"]:
        w = torch.nan_to_num(w / w.sum(dim=1, keepdim=True), nan=0.0)
    return None, w * case["scale"]


def _exact_route_backward(case, s):
    """By the chain rule of the definition, from autograd in 64 bits."""
    z = s["logits"].double().requires_grad_()
    idx, here = s["idx"].long().clamp(min=0), s["idx"] >= 0
    with torch.enable_grad():
        if case["scoring"] == "sigmoid":
            w = torch.sigmoid(z).gather(1, idx)
        else:
            lowest = torch.full_like(z, -1e300)
            w = torch.softmax(torch.where(z > -math.inf, z, lowest), dim=1).gather(1, idx)
        w = torch.where(here, w, torch.zeros_like(w))
        if case["renormalise"]:
            w = w / w.sum(dim=1, keepdim=True).clamp(min=1e-300)
        (g,) = torch.autograd.grad((w * s["grad"].double() * case["scale"]).sum(), z)
    return torch.nan_to_num(g, nan=0.0)


def _power_64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(x):
    """The nearest value of the scaled grid by distance, in 64 bits."""
    R, K = x.shape
    v = x.double().view(R, K // BLOCK, BLOCK)
    most = v.abs().amax(dim=2, keepdim=True)
    e = torch.floor(torch.log2(torch.where(most > 0, most, 1.0)))
    e = e + (most >= 2 * _power_64(e)) - (most < _power_64(e)).double()        # (a logarithm next to a whole number)
    scale = _power_64((e - 2).clamp(-127, 127))
    a = v.abs() / scale
    best, far = torch.zeros_like(a), a.clone()                              # 0, and how far it is
    for k, value in enumerate(GRID[1:], 1):
        d = (a - value).abs()
        closer = (d < far) if k % 2 else (d <= far)                          # of two as near, the even code
        best, far = torch.where(closer, torch.full_like(best, value), best), torch.where(closer, d, far)
    return (torch.sign(v) * best * scale).view(R, K)


def _exact_decode(codes, scales):
    lo, hi = codes % 16, codes // 16
    c = torch.stack([lo, hi], dim=-1).flatten(-2).long()
    m, e = c % 2, (c // 2) % 4
    v = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * _power_64(e - 1)) * (1 - 2 * (c // 8)).double()
    return v * _power_64(scales.long() - 127).repeat_interleave(BLOCK, dim=-1)


def _exact_product(x, matrices, off):
    """Expert by expert."""
    ends = off.tolist()
    y = torch.zeros(x.shape[0], matrices[0].shape[1], dtype=torch.float64, device=DEVICE)
    for e, (a, b) in enumerate(zip(ends[:-1], ends[1:])):
        if b > a:
            y[a:b] = x[a:b] @ _exact_decode(matrices[0][e], matrices[1][e]).T
    return y


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "route":
        return _exact_route(case, s["logits"], s["bias"])
    if kind == "route_backward":
        return _exact_route_backward(case, s)
    if kind in ("combine", "combine_backward"):
        T, topk, H = case["tokens"], case["topk"], case["hidden"]
        w = torch.where(s["idx"] < 0, 0.0, s["weights"].double())
        rows = s["rows"].view(T, topk, H)
        if kind == "combine":
            out = torch.zeros(T, H, dtype=torch.float64, device=DEVICE) if s["base"] is None else s["base"].double()
            for k in range(topk):
                out += w[:, k:k + 1] * rows[:, k].double()
            return out
        g = s["grad"].double()
        grad_rows = torch.empty(T, topk, H, dtype=torch.float64, device=DEVICE)
        grad_weights = torch.empty(T, topk, dtype=torch.float64, device=DEVICE)
        for k in range(topk):
            grad_rows[:, k] = w[:, k:k + 1] * g
            grad_weights[:, k] = (rows[:, k].double() * g).sum(dim=1) * (s["idx"][:, k] >= 0)
        return grad_rows.view(T * topk, H), grad_weights
    if kind == "wire":
        return _exact_values(s["x"])
    x = _exact_decode(s["codes"], s["scales"])
    if kind == "product":
        return _exact_product(x, s["w"], s["off"])
    h = _exact_product(x, s["up"], s["off"]).to(s["hidden"].dtype).double()      # (the operators meet in the layer's type)
    g, u = h.chunk(2, dim=1)
    return _exact_product(_exact_values((g * torch.sigmoid(g) * u).float()), s["down"], s["off"])
