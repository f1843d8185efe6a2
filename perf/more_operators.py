"""The work that the mixture-of-experts operators' speed is measured by: a layer of experts whose weights are held in
NVFP4 (packed nibbles, E4M3 group codes, one global scale a matrix), what chooses its experts, and what comes between
the gradients and the optimizer.

* ``route``           the k largest of softmax(logits) for each token, ties to the lowest index, with their weights;
* ``route_backward``  the gradient of those weights with respect to the logits;
* ``experts``         y_t = sum_j w_tj D_e (act(G_e x_t) * (U_e x_t)) with e = ids[t, j] (outside [0, experts): none);
* ``backward``        the gradients of ``experts`` with respect to x and the weights w;
* ``clip``            the norm over many gradients, and the gradients scaled to a largest norm.

``own`` chooses between elementary torch operations in 32 bits and the package's kernels.
"""
from __future__ import annotations

import math

import torch

own = False

BF16, F32, F64, U8, I32 = torch.bfloat16, torch.float32, torch.float64, torch.uint8, torch.int32
TYPES = {"bf16": BF16, "f32": F32}
ACTIVATIONS = {"silu": 0, "gelu_tanh": 1}


def listed():
    return [
        # the router of a layer for one decoding token: latency
        {"name": "route_token", "kind": "route", "tokens": 1, "experts": 64, "k": 8, "type": "f32", "renormalize": True,
         "masked": False, "pad": 0},
        # a large prefill batch over many experts, rows of a wider buffer
        {"name": "route_prefill", "kind": "route", "tokens": 16384, "experts": 256, "k": 8, "type": "bf16",
         "renormalize": True, "masked": False, "pad": 16},
        # odd sizes, experts switched off and padding tokens without any, weights that are not renormalized
        {"name": "route_backward_ragged", "kind": "route_backward", "tokens": 509, "experts": 61, "k": 3, "type": "f32",
         "renormalize": False, "masked": True, "pad": 3},
        # a training batch
        {"name": "route_backward_train", "kind": "route_backward", "tokens": 16384, "experts": 128, "k": 8,
         "type": "bf16", "renormalize": True, "masked": False, "pad": 0},
        # one decoding token of one request: latency, and one pass over eight experts' weights
        {"name": "experts_token", "kind": "experts", "tokens": 1, "n": 4096, "inner": 2048, "experts": 64, "k": 8,
         "activation": "silu", "skew": 0.5, "pad": 0},
        # a decoding batch of 16 requests: most experts have a token or two
        {"name": "experts_decode", "kind": "experts", "tokens": 16, "n": 4096, "inner": 2048, "experts": 64, "k": 8,
         "activation": "silu", "skew": 0.5, "pad": 0},
        # a short prompt, odd sizes, padded rows, uneven experts, slots that have none
        {"name": "experts_ragged", "kind": "experts", "tokens": 517, "n": 2064, "inner": 1360, "experts": 24, "k": 3,
         "activation": "gelu_tanh", "skew": 1.0, "pad": 24},
        # a large prefill batch
        {"name": "experts_prefill", "kind": "experts", "tokens": 4096, "n": 4096, "inner": 2048, "experts": 64, "k": 8,
         "activation": "silu", "skew": 0.5, "pad": 0},
        # the smallest layer and a short sequence trained through
        {"name": "backward_small", "kind": "backward", "tokens": 96, "n": 1024, "inner": 512, "experts": 8, "k": 2,
         "activation": "silu", "skew": 0.5, "pad": 8},
        # a training batch through a layer of few wide experts
        {"name": "backward_train", "kind": "backward", "tokens": 2048, "n": 4096, "inner": 14336, "experts": 8, "k": 2,
         "activation": "silu", "skew": 0.5, "pad": 0},
        # the adapters' gradients of one small layer
        {"name": "clip_small", "kind": "clip", "tensors": 14, "largest": 65536, "type": "bf16", "scale": 1e-3},
        # every adapter's gradients of a deep model, in 32 bits
        {"name": "clip_deep", "kind": "clip", "tensors": 1120, "largest": 917504, "type": "f32", "scale": 1e-4},
    ]


def _log(rng, lo, hi, step=1):
    """A whole number spread over the logarithm of [lo, hi], a multiple of step."""
    v = lo * (hi / lo) ** rng.random()
    return max(step, min(hi // step * step, int(v / step + 0.5) * step))


def draw(rng):
    kind = rng.choice(["route", "route_backward", "experts", "experts", "experts", "experts", "backward", "backward",
                       "clip"])
    pad = rng.choice([0, 0, 8, 24, 64])
    if kind in ("route", "route_backward"):
        experts = _log(rng, 4, 512)
        return {"kind": kind, "tokens": _log(rng, 1, 16384), "experts": experts, "k": min(experts, _log(rng, 1, 16)),
                "type": rng.choice(["bf16", "f32"]), "renormalize": rng.random() < 0.5, "masked": rng.random() < 0.5,
                "pad": rng.choice([0, 3, 16])}
    if kind == "clip":
        return {"kind": kind, "tensors": _log(rng, 1, 1000), "largest": _log(rng, 1000, 900000),
                "type": rng.choice(["bf16", "f32"]), "scale": 10.0 ** rng.uniform(-6, 1)}
    n = _log(rng, 512, 8192, rng.choice([16, 64, 512]))
    inner = _log(rng, 256, 4096, rng.choice([16, 64, 256]))
    experts = _log(rng, 4, max(4, min(128, (1 << 29) // (n * inner))))
    k = min(experts, _log(rng, 1, 8))
    most = (1 << 38) // (n * inner * k)  # slots times weights no more than the largest listed ones
    if kind == "experts":
        tokens = _log(rng, 1, max(1, min(4096, most)))
    else:
        tokens = _log(rng, 16, max(16, min(4096, most // 2)))
    return {"kind": kind, "tokens": tokens, "n": n, "inner": inner, "experts": experts, "k": k,
            "activation": rng.choice(["silu", "silu", "gelu_tanh"]), "skew": rng.choice([0.0, 0.5, 1.0]), "pad": pad}


def _clip_sizes(case):
    """Sizes of the gradients: of adapters A [rank, n] and B [m, rank] of several ranks and widths, and a few
    vectors."""
    sizes = []
    for i in range(case["tensors"]):
        part = (1.0, 0.25, 0.5, 0.875, 0.125, 0.001, 0.3)[i % 7]
        sizes.append(max(1, int(case["largest"] * part) - (i % 5 == 3)))
    return sizes


def work(case):
    kind = case["kind"]
    if kind == "clip":
        size = 2 if case["type"] == "bf16" else 4
        count = sum(_clip_sizes(case))
        return {"bytes": 2 * size * count + 4, "flops": 3 * count}
    t, e, k = case["tokens"], case["experts"], case["k"]
    if kind in ("route", "route_backward"):
        size = 2 if case["type"] == "bf16" else 4
        if kind == "route":
            return {"bytes": t * (e * size + 8 * k), "flops": t * e * 4}
        return {"bytes": t * (2 * e * size + 12 * k), "flops": t * e * 4}
    n, inner = case["n"], case["inner"]
    used = max(1, round(e * (1.0 - (1.0 - k / e) ** t)))  # experts that some token is on
    weights = used * 3 * n * inner * 9 // 16
    if kind == "experts":
        return {"bytes": weights + 4 * t * n + 8 * t * k, "flops": 6 * t * k * n * inner}
    # g and u made again, dh, and the two products of dx
    return {"bytes": weights + 6 * t * n + 12 * t * k, "flops": 10 * t * k * n * inner}


# ---------------------------------------------------------------- inputs
def _dev():
    return torch.device("cuda", 0)


def _gen(seed, *salt):
    g = torch.Generator(device=_dev())
    g.manual_seed((seed * 1000003 + sum((i + 1) * 7919 * int(v) for i, v in enumerate(salt))) % (1 << 62))
    return g


def _rows(tokens, cols, pad, dtype=BF16):
    """An uninitialised [tokens, cols] view of rows that are pad or a few more elements longer (whole 16 bytes of
    bf16)."""
    ld = cols + pad
    if dtype == BF16 and (pad or cols % 8):
        ld = (ld + 7) // 8 * 8
    return torch.empty(tokens, ld, dtype=dtype, device=_dev())[:, :cols]


def _activations(tokens, n, pad, g):
    """Channel magnitudes spread log-normally with a few outlier channels, as a layer's inputs have."""
    mag = torch.exp(0.5 * torch.randn(n, generator=g, device=_dev()))
    outliers = torch.randint(n, (max(1, n // 512),), generator=g, device=_dev())
    mag[outliers] *= 10.0
    x = _rows(tokens, n, pad)
    x[:] = (torch.randn(tokens, n, generator=g, device=_dev()) * mag).to(BF16)
    return x


def _quantized(experts, m, n, g):
    """Weight matrices with heavy tails rounded to NVFP4: packed nibbles, E4M3 codes, a global scale each."""
    packed = torch.empty(experts, m, n // 2, dtype=U8, device=_dev())
    codes = torch.empty(experts, m, n // 16, dtype=U8, device=_dev())
    sg = torch.empty(experts, dtype=F32, device=_dev())
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=_dev())
    for e in range(experts):
        w = torch.randn(m, n, generator=g, device=_dev())
        w *= torch.exp(0.5 * torch.randn(m, 1, generator=g, device=_dev())) / math.sqrt(n)
        sg[e] = w.abs().max() / 2688.0
        grp = w.reshape(m, n // 16, 16)
        c = (grp.abs().amax(2) / (6.0 * sg[e])).to(torch.float8_e4m3fn).view(U8).clamp(1, 126)
        scale = c.view(torch.float8_e4m3fn).to(F32) * sg[e]
        nib = torch.bucketize((grp.abs() / scale[:, :, None]).reshape(m, n), edges, out_int32=True).to(U8)
        nib |= (w < 0).to(U8) << 3
        packed[e] = nib[:, 0::2] | (nib[:, 1::2] << 4)
        codes[e] = c
    return packed, codes, sg


def _logits(case, g, skew):
    """Router scores: some experts liked better than others.  Masked: a few experts are off (-inf) and some rows, of
    padding, have none."""
    t, e = case["tokens"], case["experts"]
    v = 1.5 * torch.randn(t, e, generator=g, device=_dev()) + skew * torch.randn(e, generator=g, device=_dev())
    if case.get("masked"):
        v[:, torch.rand(e, generator=g, device=_dev()) < 0.1] = -math.inf
        v[torch.rand(t, generator=g, device=_dev()) < 0.05] = -math.inf
    return v


def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case}
    if kind == "clip":
        g = _gen(seed, case["tensors"], case["largest"])
        sizes = _clip_sizes(case)
        whole = torch.randn(sum(sizes), generator=g, device=_dev())
        s["grads"], at = [], 0
        for i, size in enumerate(sizes):
            level = case["scale"] * math.exp(math.sin(3.0 * i + seed))
            s["grads"].append((whole[at:at + size] * level).to(TYPES[case["type"]]))
            at += size
        s["max_norm"] = 0.5 * case["scale"] * math.sqrt(sum(sizes))
        # the scaled gradients go to places in one buffer, each a whole number of 64 elements
        room = [(size + 63) // 64 * 64 for size in sizes]
        s["buffer"] = torch.zeros(sum(room), dtype=TYPES[case["type"]], device=_dev())
        s["out"] = [part[:size] for part, size in zip(s["buffer"].split(room), sizes)]
        s["norm"] = torch.empty(1, dtype=F32, device=_dev())
        if own:
            import paper_2608_28113_gb300 as hs
            s["lists"] = hs.hscale_tensors(s["grads"]), hs.hscale_tensors(s["out"])
            s["ws"] = torch.empty(hs.hscale_grad_norm_workspace_bytes(), dtype=U8, device=_dev())
        return s
    t, e, k = case["tokens"], case["experts"], case["k"]
    g = _gen(seed, t, e, k, case.get("n", 0), case.get("inner", 0))
    if kind in ("route", "route_backward"):
        s["logits"] = _rows(t, e, case["pad"], TYPES[case["type"]])
        s["logits"][:] = _logits(case, g, 0.5).to(TYPES[case["type"]])
        if kind == "route_backward":
            s["ids"], s["weights"] = _route(s["logits"], k, case["renormalize"])
            s["dweights"] = torch.randn(t, k, generator=g, device=_dev())
            s["dlogits"] = _rows(t, e, case["pad"], TYPES[case["type"]])
        else:
            s["ids"] = torch.empty(t, k, dtype=I32, device=_dev())
            s["weights"] = torch.empty(t, k, dtype=F32, device=_dev())
        return s
    n, inner = case["n"], case["inner"]
    s["x"] = _activations(t, n, case["pad"], g)
    s["ids"], s["weights"] = _route(_logits(case, g, case["skew"]), k, True)
    if case["skew"] == 1.0:  # tokens dropped by a full expert
        s["ids"] = torch.where(torch.rand(t, k, generator=g, device=_dev()) < 0.03, -1, s["ids"]).to(I32)
    s["gate"], s["up"] = _quantized(e, inner, n, g), _quantized(e, inner, n, g)
    s["down"] = _quantized(e, n, inner, g)
    if kind == "backward":
        s["dy"] = _rows(t, n, case["pad"])
        s["dy"][:] = (torch.randn(t, n, generator=g, device=_dev()) * 1e-2).to(BF16)
        s["dx"], s["dweights"] = _rows(t, n, case["pad"]), torch.empty_like(s["weights"])
    else:
        s["y"] = _rows(t, n, case["pad"])
    if own:
        import paper_2608_28113_gb300 as hs
        if kind == "experts":
            nbytes = hs.hscale_experts_workspace_bytes(t, k, n, inner, e)
        else:
            nbytes = hs.hscale_experts_backward_workspace_bytes(t, k, n, inner, e)
        s["ws"] = torch.empty(max(256, nbytes), dtype=U8, device=_dev())
    return s


# ---------------------------------------------------------------- one pass
def _route(logits, k, renormalize):
    v = logits.to(F32)
    top = v.amax(1, keepdim=True)
    p = torch.exp(v - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(1, keepdim=True)
    value, index = torch.sort(v, dim=1, descending=True, stable=True)
    some = value[:, :k] > -math.inf
    ids = torch.where(some, index[:, :k], -1).to(I32)
    picked = torch.where(some, p.gather(1, index[:, :k]), 0.0)
    if renormalize:
        total = picked.sum(1, keepdim=True)
    return ids, torch.where(total > 0, picked / total, 0.0)


def _route_backward(s):
    case = s["case"]
    v, ids = s["logits"].to(F32), s["ids"].to(torch.int64)
    on = ids >= 0
    w = torch.where(on, s["weights"], 0.0)
    dw = torch.where(on, s["dweights"], 0.0)
    mean = (w * dw).sum(1, keepdim=True)
    if case["renormalize"]:
        out = torch.zeros_like(v)
        return out.scatter_add(1, ids.clamp(min=0), torch.where(on, w * (dw - mean), 0.0)).to(s["logits"].dtype)
    top = v.amax(1, keepdim=True)
    p = torch.exp(v - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(1, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    spread = torch.zeros_like(v).scatter_add(1, ids.clamp(min=0), dw)
    return (p * (spread - mean)).to(s["logits"].dtype)


def _weight(w, e):
    """Expert e's NVFP4 matrix in 32 bits."""
    packed, codes, sg = w[0][e], w[1][e], w[2][e]
    m, half = packed.shape
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                        dtype=F32, device=packed.device)
    nib = torch.stack((packed & 15, packed >> 4), dim=2).reshape(m, 2 * half)
    scale = codes.view(torch.float8_e4m3fn).to(F32) * sg
    return grid[nib.to(I32)] * scale.repeat_interleave(16, dim=1)


def _act(g, kind):
    """The activation and its derivative."""
    if kind == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        return g * sig, sig * (1.0 + g * (1.0 - sig))
    c = math.sqrt(2.0 / math.pi)
    th = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * c * (1.0 + 3 * 0.044715 * g * g)


def _plain_experts(s):
    case, ids = s["case"], s["ids"]
    x = s["x"].to(F32)
    y = torch.zeros_like(x)
    for e in ids.unique().tolist():
        if e < 0:
            continue
        rows, slot = (ids == e).nonzero(as_tuple=True)
        xe = x[rows]
        a, _ = _act(xe @ _weight(s["gate"], e).T, case["activation"])
        h = a * (xe @ _weight(s["up"], e).T)
        y.index_add_(0, rows, (h @ _weight(s["down"], e).T) * s["weights"][rows, slot][:, None])
    return {"y": y.to(BF16)}


def _plain_backward(s):
    case, ids = s["case"], s["ids"]
    x, dy = s["x"].to(F32), s["dy"].to(F32)
    dx, dw = torch.zeros_like(x), torch.zeros_like(s["weights"])
    for e in ids.unique().tolist():
        if e < 0:
            continue
        rows, slot = (ids == e).nonzero(as_tuple=True)
        gate, up = _weight(s["gate"], e), _weight(s["up"], e)
        xe, w = x[rows], s["weights"][rows, slot][:, None]
        g, u = xe @ gate.T, xe @ up.T
        a, slope = _act(g, case["activation"])
        dh = dy[rows] @ _weight(s["down"], e)
        dw[rows, slot] = (dh * a * u).sum(1)
        dx.index_add_(0, rows, (w * dh * u * slope) @ gate + (w * dh * a) @ up)
    return {"dx": dx.to(BF16), "dweights": dw}


def _plain_clip(s):
    total = torch.zeros((), dtype=F64, device=_dev())
    for v in s["grads"]:
        v = v.to(F32)
        total += (v * v).sum(dtype=F64)
    norm = torch.sqrt(total).to(F32)
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    for v, out in zip(s["grads"], s["out"]):
        out.copy_(v.to(F32) * factor)
    return {"norm": norm.reshape(1), "grads": s["buffer"]}


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        if kind == "route":
            ids, weights = _route(s["logits"], case["k"], case["renormalize"])
            return {"ids": ids, "weights": weights}
        if kind == "route_backward":
            return {"dlogits": _route_backward(s)}
        if kind == "clip":
            return _plain_clip(s)
        return _plain_experts(s) if kind == "experts" else _plain_backward(s)
    import paper_2608_28113_gb300 as hs
    if kind == "route":
        hs.hscale_route(s["logits"], s["ids"], s["weights"], case["renormalize"])
        return {"ids": s["ids"], "weights": s["weights"]}
    if kind == "route_backward":
        hs.hscale_route_backward(s["logits"], s["ids"], s["weights"], s["dweights"], case["renormalize"], s["dlogits"])
        return {"dlogits": s["dlogits"]}
    if kind == "clip":
        hs.hscale_grad_clip(s["lists"][0], s["max_norm"], s["norm"], s["lists"][1], s["ws"])
        return {"norm": s["norm"], "grads": s["buffer"]}
    act = ACTIVATIONS[case["activation"]]
    if kind == "experts":
        hs.hscale_experts(s["x"], s["ids"], s["weights"], s["gate"], s["up"], s["down"], act, s["y"], s["ws"])
        return {"y": s["y"]}
    hs.hscale_experts_backward(s["dy"], s["x"], s["ids"], s["weights"], s["gate"], s["up"], s["down"], act, s["dx"],
                               s["dweights"], s["ws"])
    return {"dx": s["dx"], "dweights": s["dweights"]}


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_weight(w, e):
    p = w[0][e].to(torch.int64)
    m, n = p.shape[0], 2 * p.shape[1]
    nib = torch.empty(m, n, dtype=torch.int64, device=p.device)
    nib[:, 0::2], nib[:, 1::2] = p % 16, p // 16
    mag, sign = nib % 8, 1.0 - 2.0 * (nib // 8).to(F64)
    exp, man = mag // 2, (mag % 2).to(F64)
    val = torch.where(exp == 0, 0.5 * man, torch.exp2((exp - 1).to(F64)) * (1.0 + 0.5 * man)) * sign
    c = w[1][e].to(torch.int64)
    ce, cm = c // 8, (c % 8).to(F64)
    scale = torch.where(ce == 0, cm * 2.0 ** -9, torch.exp2((ce - 7).to(F64)) * (1.0 + cm / 8.0)) * w[2][e].to(F64)
    return (val.reshape(m, n // 16, 16) * scale[:, :, None]).reshape(m, n)


def _exact_act(g, kind):
    if kind == "silu":
        return g / (1.0 + torch.exp(-g))
    return g / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)))


def _exact_slope(g, kind):
    """The derivative from act = g s(q(g)), s the logistic function."""
    if kind == "silu":
        q, dq = g, torch.ones_like(g)
    else:
        c = 2.0 * math.sqrt(2.0 / math.pi)
        q, dq = c * (g + 0.044715 * g ** 3), c * (1.0 + 0.134145 * g ** 2)
    sig, rest = 1.0 / (1.0 + torch.exp(-q)), 1.0 / (1.0 + torch.exp(q))
    return sig + g * dq * sig * rest


def _exact_route(s):
    v, k = s["logits"].to(F64), s["case"]["k"]
    left, index = v.clone(), torch.arange(v.shape[1], device=v.device)
    ids, value = [], []
    for _ in range(k):
        best = left.amax(1, keepdim=True)
        at = torch.where(left == best, index, v.shape[1]).amin(1, keepdim=True)
        ids.append(torch.where(best > -math.inf, at, -1))
        value.append(best)
        left = torch.where(index == at, -math.inf, left)
    ids, value = torch.cat(ids, 1), torch.cat(value, 1)
    logsum = torch.logsumexp(value if s["case"]["renormalize"] else v, 1, keepdim=True)
    return {"ids": ids.to(I32), "weights": torch.where(ids >= 0, torch.exp(value - logsum), 0.0)}


def _exact_route_backward(s):
    v, ids, w, dw = s["logits"].to(F64), s["ids"], s["weights"].to(F64), s["dweights"].to(F64)
    out = torch.zeros_like(v)
    rows = torch.arange(v.shape[0], device=v.device)
    mean = torch.zeros(v.shape[0], dtype=F64, device=v.device)
    for j in range(ids.shape[1]):
        mean += torch.where(ids[:, j] >= 0, w[:, j] * dw[:, j], 0.0)
    if not s["case"]["renormalize"]:
        p = torch.softmax(v, 1)
        p = torch.where(torch.isnan(p), 0.0, p)
        out = -p * mean[:, None]
    for j in range(ids.shape[1]):
        on = ids[:, j] >= 0
        r, c = rows[on], ids[on, j].to(torch.int64)
        if s["case"]["renormalize"]:
            out[r, c] = w[on, j] * (dw[on, j] - mean[on])
        else:
            out[r, c] += p[r, c] * dw[on, j]
    return {"dlogits": out}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "route":
        return _exact_route(s)
    if kind == "route_backward":
        return _exact_route_backward(s)
    if kind == "clip":
        norm = math.sqrt(sum(float((v.to(F64) ** 2).sum()) for v in s["grads"]))
        factor = min(1.0, s["max_norm"] / norm) if norm > 0 else 1.0
        parts = [torch.nn.functional.pad(v.to(F64) * factor, (0, -v.numel() % 64)) for v in s["grads"]]
        return {"norm": torch.tensor([norm], dtype=F64, device=_dev()), "grads": torch.cat(parts)}
    x, ids, w = s["x"].to(F64), s["ids"], s["weights"].to(F64)
    if kind == "experts":
        out = torch.zeros_like(x)
    else:
        dy, out, dw = s["dy"].to(F64), torch.zeros_like(x), torch.zeros_like(w)
    for e in ids.unique().tolist():
        if e < 0:
            continue
        gate, up, down = _exact_weight(s["gate"], e), _exact_weight(s["up"], e), _exact_weight(s["down"], e)
        for j in range(case["k"]):
            rows = (ids[:, j] == e).nonzero().squeeze(1)
            if rows.numel() == 0:
                continue
            g, u = x[rows] @ gate.T, x[rows] @ up.T
            act = _exact_act(g, case["activation"])
            if kind == "experts":
                out[rows] += w[rows, j, None] * ((act * u) @ down.T)
                continue
            dh = dy[rows] @ down
            dw[rows, j] = (act * u * dh).sum(1)
            out[rows] += w[rows, j, None] * ((dh * u * _exact_slope(g, case["activation"])) @ gate + (dh * act) @ up)
    return {"y": out} if kind == "experts" else {"dx": out, "dweights": dw}
