"""The work that the adapter operators' speed is measured by: three operators around a projection whose
weights are held in NVFP4 (packed nibbles, E4M3 group codes, one global scale).

* ``checkpoint``  activations kept in 8 bits between the passes of a training step: blocks of 32 channels
                  with a power of two as their scale, INT8 or E4M3 elements; saved, then loaded again;
* ``project``     y_t = W x_t + alpha_a B_a (A_a x_t) with a = adapter of token t (none: the first term
                  alone), W the NVFP4 weight, A_a and B_a the low-rank adapters of many requests;
* ``backward``    the gradients dx, dA, dB of ``project``, with x taken from its 8-bit checkpoint.

``own`` chooses between elementary torch operations in 32 bits and the package's kernels.
"""
from __future__ import annotations

import math

import torch

own = False

BF16, F32, F64, U8, I32 = torch.bfloat16, torch.float32, torch.float64, torch.uint8, torch.int32
FORMATS = {"int8": 0, "e4m3": 1}
BLOCK = 32


def listed():
    return [
        # the input of a 4096-wide projection kept over one calibration-sized chunk of tokens
        {"name": "checkpoint_attention", "kind": "checkpoint", "tokens": 8192, "n": 4096, "format": "int8", "pad": 0},
        # a short sequence through an MLP's down projection, E4M3 elements, rows of a wider buffer
        {"name": "checkpoint_ragged", "kind": "checkpoint", "tokens": 517, "n": 14336, "format": "e4m3", "pad": 16},
        # one token of one request: a call whose cost is latency and one pass over the weights
        {"name": "project_token", "kind": "project", "tokens": 1, "m": 4096, "n": 4096, "adapters": 8, "rank": 16,
         "order": "mixed", "pad": 0},
        # a decoding batch, one token each of 16 requests, on the widest MLP matrix
        {"name": "project_decode_wide", "kind": "project", "tokens": 16, "m": 28672, "n": 8192, "adapters": 16,
         "rank": 16, "order": "mixed", "pad": 0},
        # a fuller decoding batch over many adapters
        {"name": "project_decode_many", "kind": "project", "tokens": 64, "m": 14336, "n": 4096, "adapters": 64,
         "rank": 16, "order": "mixed", "pad": 0},
        # odd sizes and padded rows, a few tokens of requests without an adapter among them
        {"name": "project_ragged", "kind": "project", "tokens": 37, "m": 3001, "n": 3216, "adapters": 5, "rank": 8,
         "order": "mixed", "pad": 24},
        # a chunk of prefill of four requests through a down projection
        {"name": "project_chunk", "kind": "project", "tokens": 512, "m": 4096, "n": 14336, "adapters": 4, "rank": 32,
         "order": "requests", "pad": 0},
        # a large prefill batch of 16 requests through an up projection
        {"name": "project_prefill", "kind": "project", "tokens": 8192, "m": 14336, "n": 4096, "adapters": 16,
         "rank": 16, "order": "requests", "pad": 0},
        # fine-tuning one adapter on an attention projection
        {"name": "backward_attention", "kind": "backward", "tokens": 8192, "m": 4096, "n": 4096, "adapters": 1,
         "rank": 16, "order": "one", "format": "int8", "pad": 0},
        # many small adapters trained together on a narrow key projection, tokens in any order
        {"name": "backward_mixed", "kind": "backward", "tokens": 2048, "m": 1024, "n": 4096, "adapters": 32,
         "rank": 8, "order": "mixed", "format": "int8", "pad": 0},
        # four larger adapters on a down projection
        {"name": "backward_wide", "kind": "backward", "tokens": 4096, "m": 4096, "n": 14336, "adapters": 4,
         "rank": 64, "order": "requests", "format": "e4m3", "pad": 0},
        # the smallest layer and a short sequence: latency
        {"name": "backward_small", "kind": "backward", "tokens": 96, "m": 512, "n": 1024, "adapters": 2, "rank": 16,
         "order": "requests", "format": "int8", "pad": 8},
    ]


def _log(rng, lo, hi, step=1):
    """A whole number spread over the logarithm of [lo, hi], a multiple of step."""
    v = lo * (hi / lo) ** rng.random()
    return max(step, min(hi // step * step, int(v / step + 0.5) * step))


def draw(rng):
    kind = rng.choice(["checkpoint", "project", "project", "project", "backward", "backward"])
    pad = rng.choice([0, 0, 8, 24, 64])
    if kind == "checkpoint":
        n = _log(rng, 256, 28672, rng.choice([1, 16, 64]))
        return {"kind": kind, "tokens": _log(rng, 1, min(65536, (1 << 28) // n)), "n": n,
                "format": rng.choice(["int8", "e4m3"]), "pad": pad}
    n = _log(rng, 256, 14336, rng.choice([16, 64, 512]))
    m = _log(rng, 64, 28672, rng.choice([1, 8, 128]))
    rank = rng.choice([8, 16, 16, 32, 64])
    if kind == "project":
        tokens = _log(rng, 1, min(8192, max(1, 8192 * 4096 * 4096 // (n * m))))
        adapters = _log(rng, 1, 64)
        return {"kind": kind, "tokens": tokens, "m": m, "n": n, "adapters": adapters, "rank": rank,
                "order": rng.choice(["requests", "requests", "mixed"]), "pad": pad}
    tokens = _log(rng, 16, min(8192, max(16, 4096 * 4096 * 4096 // (n * m))))
    adapters = _log(rng, 1, 32)
    return {"kind": kind, "tokens": tokens, "m": m, "n": n, "adapters": adapters, "rank": rank,
            "order": "one" if adapters == 1 else rng.choice(["requests", "requests", "mixed"]),
            "format": rng.choice(["int8", "e4m3"]), "pad": pad}


def work(case):
    t, n = case["tokens"], case["n"]
    blocks = (n + BLOCK - 1) // BLOCK
    if case["kind"] == "checkpoint":
        # save: x in, elements and scales out; load: those in, x out
        return {"bytes": 2 * (2 * t * n + t * n + t * blocks), "flops": 4 * t * n}
    m, r = case["m"], case["rank"]
    used = min(case["adapters"], t)
    weight = m * n // 2 + m * n // 16
    if case["kind"] == "project":
        return {"bytes": weight + 2 * t * (m + n) + 2 * used * r * (m + n) + 4 * t,
                "flops": 2 * t * m * n + 2 * t * r * (m + n)}
    # dx, the products dy B and x A^T, and the two gradients
    return {"bytes": weight + 2 * t * (m + n) + t * (n + blocks) + 2 * used * r * (m + n) +
            2 * case["adapters"] * r * (m + n) + 4 * t,
            "flops": 2 * t * m * n + 6 * t * r * (m + n)}


# ---------------------------------------------------------------- inputs
def _dev():
    return torch.device("cuda", 0)


def _gen(seed, *salt):
    g = torch.Generator(device=_dev())
    g.manual_seed((seed * 1000003 + sum((i + 1) * 7919 * int(v) for i, v in enumerate(salt))) % (1 << 62))
    return g


def _rows(tokens, cols, pad):
    """An uninitialised bf16 [tokens, cols] view of rows that are pad or a few more elements longer."""
    ld = cols + pad if pad == 0 else (cols + pad + 7) // 8 * 8
    if pad == 0 and cols % 8:
        ld = (cols + 7) // 8 * 8
    return torch.empty(tokens, ld, dtype=BF16, device=_dev())[:, :cols]


def _activations(tokens, n, pad, g):
    """Channel magnitudes spread log-normally with a few outlier channels, as a layer's inputs have."""
    mag = torch.exp(torch.randn(n, generator=g, device=_dev()))
    outliers = torch.randint(n, (max(1, n // 512),), generator=g, device=_dev())
    mag[outliers] *= 20.0
    x = _rows(tokens, n, pad)
    for t in range(0, tokens, 4096):
        part = torch.randn(min(4096, tokens - t), n, generator=g, device=_dev())
        x[t:t + 4096] = (part * mag).to(BF16)
    return x


def _quantized(m, n, g):
    """A heavy-tailed weight matrix rounded to NVFP4: packed nibbles, E4M3 codes, global scale."""
    w = torch.randn(m, n, generator=g, device=_dev())
    w *= torch.exp(0.5 * torch.randn(m, n, generator=g, device=_dev())) * 0.02
    sg = (w.abs().max() / 2688.0).reshape(1)
    grp = w.reshape(m, n // 16, 16)
    codes = (grp.abs().amax(2) / (6.0 * sg)).to(torch.float8_e4m3fn).view(U8).clamp(1, 126)
    scale = codes.view(torch.float8_e4m3fn).to(F32) * sg
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=_dev())
    nib = torch.bucketize((grp.abs() / scale[:, :, None]).reshape(m, n), edges, out_int32=True).to(U8)
    nib |= (w < 0).to(U8) << 3
    packed = nib[:, 0::2] | (nib[:, 1::2] << 4)
    return packed.contiguous(), codes.contiguous(), sg


def _adapter_of(case, g):
    """The adapter of each token: tokens of one request side by side, or in any order; one in sixteen
    requests (tokens, where they are mixed) has none."""
    t, count = case["tokens"], case["adapters"]
    if case["order"] == "one":
        return torch.zeros(t, dtype=I32, device=_dev())
    if case["order"] == "mixed":
        ids = torch.randperm(max(t, count), generator=g, device=_dev())[:t] % count
        return torch.where(torch.rand(t, generator=g, device=_dev()) < 1 / 16, -1, ids).to(I32)
    cuts = torch.randint(t + 1, (count - 1,), generator=g, device=_dev()).sort().values
    ids = torch.searchsorted(cuts, torch.arange(t, device=_dev()), right=True)
    none = torch.rand(count, generator=g, device=_dev()) < 1 / 16
    return torch.where(none[ids], -1, ids).to(I32)


def _save(x, fmt):
    """The elements and scale bytes of a checkpoint, in elementary operations."""
    t, n = x.shape
    blocks = (n + BLOCK - 1) // BLOCK
    v = torch.zeros(t, blocks * BLOCK, dtype=F32, device=x.device)
    v[:, :n] = x
    v = v.reshape(t, blocks, BLOCK)
    amax = v.abs().amax(2)
    mant, exp = torch.frexp(amax)  # amax = mant 2^exp, mant in [0.5, 1)
    if fmt == "int8":
        e = exp - 7
    else:
        e = exp - 9 + (mant > 0.875)  # 448 = 0.875 * 2^9
    e = torch.where(amax > 0, e, -124).clamp(-124, 124).to(I32)
    inv = ((127 - e) << 23).view(F32)
    v = v * inv[:, :, None]
    if fmt == "int8":
        q = v.round().clamp(-127, 127).to(torch.int8).view(U8)
    else:
        q = v.to(torch.float8_e4m3fn).view(U8)
    return q.reshape(t, blocks * BLOCK)[:, :n], (e + 127).to(U8)


def _load(q, scales, fmt, dtype):
    n = q.shape[1]
    kind = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    s = (scales.to(I32) << 23).view(F32).to(dtype)
    return q.contiguous().view(kind).to(dtype) * s.repeat_interleave(BLOCK, dim=1)[:, :n]


def prepare(case, seed):
    dev, t, n, pad = _dev(), case["tokens"], case["n"], case["pad"]
    g = _gen(seed, t, n, case.get("m", 0), case.get("rank", 0))
    s = {"case": case}
    x = _activations(t, n, pad, g)
    if case["kind"] == "checkpoint":
        s["x"] = x
        if own:
            s["q"] = torch.empty(t, n, dtype=U8, device=dev)
            s["scales"] = torch.empty(t, (n + BLOCK - 1) // BLOCK, dtype=U8, device=dev)
            s["out"] = _rows(t, n, pad)
        return s
    m, r, count = case["m"], case["rank"], case["adapters"]
    s["packed"], s["codes"], s["sg"] = _quantized(m, n, g)
    s["a"] = (torch.randn(count, r, n, generator=g, device=dev) / math.sqrt(n)).to(BF16)
    s["b"] = (torch.randn(count, m, r, generator=g, device=dev) * 0.02).to(BF16)
    s["alpha"] = 0.5 + 2.0 * torch.rand(count, generator=g, device=dev)
    s["ids"] = _adapter_of(case, g)
    if case["kind"] == "project":
        s["x"] = x
    else:
        q, scales = _save(x, case["format"])
        s["q"], s["scales"] = q.contiguous(), scales.contiguous()
        dy = _rows(t, m, pad)
        dy[:] = (torch.randn(t, m, generator=g, device=dev) * 1e-2).to(BF16)
        s["dy"] = dy
    if own:
        import paper_2608_28113_gb300 as hs
        if case["kind"] == "project":
            s["y"] = _rows(t, m, pad)
            nbytes = hs.hscale_project_workspace_bytes(t, m, n, count, r)
        else:
            s["dx"] = _rows(t, n, pad)
            s["da"], s["db"] = torch.empty_like(s["a"]), torch.empty_like(s["b"])
            nbytes = hs.hscale_project_backward_workspace_bytes(t, m, n, count, r)
        s["ws"] = torch.empty(max(256, nbytes), dtype=U8, device=dev)
    return s


# ---------------------------------------------------------------- one pass
def _weight(packed, codes, sg):
    """The NVFP4 weight in 32 bits."""
    m, half = packed.shape
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                        dtype=F32, device=packed.device)
    nib = torch.stack((packed & 15, packed >> 4), dim=2).reshape(m, 2 * half)
    scale = codes.view(torch.float8_e4m3fn).to(F32) * sg
    return grid[nib.to(I32)] * scale.repeat_interleave(16, dim=1)


def _plain_project(s):
    x, ids = s["x"].to(F32), s["ids"]
    y = x @ _weight(s["packed"], s["codes"], s["sg"]).T
    for a in range(s["case"]["adapters"]):
        z = x @ s["a"][a].to(F32).T
        z = torch.where((ids == a)[:, None], z * s["alpha"][a], 0.0)
        y += z @ s["b"][a].to(F32).T
    return {"y": y.to(BF16)}


def _plain_backward(s):
    case, ids = s["case"], s["ids"]
    x = _load(s["q"], s["scales"], case["format"], F32)
    dy = s["dy"].to(F32)
    dx = dy @ _weight(s["packed"], s["codes"], s["sg"])
    da, db = torch.empty_like(s["a"]), torch.empty_like(s["b"])
    for a in range(case["adapters"]):
        wa, wb, on = s["a"][a].to(F32), s["b"][a].to(F32), (ids == a)[:, None]
        z = torch.where(on, (x @ wa.T) * s["alpha"][a], 0.0)
        dz = torch.where(on, (dy @ wb) * s["alpha"][a], 0.0)
        dx += dz @ wa
        da[a] = (dz.T @ x).to(BF16)
        db[a] = (dy.T @ z).to(BF16)
    return {"dx": dx.to(BF16), "da": da, "db": db}


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        if kind == "checkpoint":
            q, scales = _save(s["x"], case["format"])
            return {"x": _load(q, scales, case["format"], F32).to(BF16)}
        return _plain_project(s) if kind == "project" else _plain_backward(s)
    import paper_2608_28113_gb300 as hs
    if kind == "checkpoint":
        fmt = FORMATS[case["format"]]
        hs.hscale_checkpoint_save(s["x"], fmt, s["q"], s["scales"])
        hs.hscale_checkpoint_load(s["q"], s["scales"], fmt, s["out"])
        return {"x": s["out"]}
    if kind == "project":
        hs.hscale_project(s["x"], s["packed"], s["codes"], s["sg"], s["a"], s["b"], s["alpha"], s["ids"], s["y"],
                          s["ws"])
        return {"y": s["y"]}
    hs.hscale_project_backward(s["dy"], s["q"], s["scales"], FORMATS[case["format"]], s["packed"], s["codes"],
                               s["sg"], s["a"], s["b"], s["alpha"], s["ids"], s["dx"], s["da"], s["db"], s["ws"])
    return {"dx": s["dx"], "da": s["da"], "db": s["db"]}


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_checkpoint(x, fmt):
    """Each element rounded to the block's grid: steps of 2^e (INT8), or four significant bits and
    steps of 2^(e - 9) at least (E4M3), with 2^e from the block's largest magnitude."""
    t, n = x.shape
    out = torch.empty(t, n, dtype=F64, device=x.device)
    for t0 in range(0, t, 4096):
        part = x[t0:t0 + 4096].to(F64)
        rows = part.shape[0]
        full = torch.nn.functional.pad(part, (0, -n % BLOCK)).reshape(rows, -1, BLOCK)
        amax = full.abs().amax(2, keepdim=True).clamp(min=2.0 ** -133)
        top = torch.floor(torch.log2(amax))
        top = torch.where(torch.exp2(top) > amax, top - 1, torch.where(torch.exp2(top + 1) <= amax, top + 1, top))
        if fmt == "int8":
            step = torch.exp2((top - 6).clamp(min=-124))
            val = (torch.round(full / step)).clamp(-127, 127) * step
        else:
            e = (top - 8 + (amax > 1.75 * torch.exp2(top)).to(F64)).clamp(min=-124)
            mag = (full.abs() * torch.exp2(-e)).clamp(min=2.0 ** -40)
            own_exp = torch.frexp(mag)[1].to(F64) - 1
            step = torch.exp2(own_exp.clamp(min=-6) - 3)
            val = torch.round(full * torch.exp2(-e) / step) * step * torch.exp2(e)
        out[t0:t0 + rows] = val.reshape(rows, -1)[:, :n]
    return out


def _weight64(s):
    p = s["packed"].to(torch.int64)
    m, n = p.shape[0], 2 * p.shape[1]
    nib = torch.empty(m, n, dtype=torch.int64, device=p.device)
    nib[:, 0::2], nib[:, 1::2] = p % 16, p // 16
    mag, sign = nib % 8, 1.0 - 2.0 * (nib // 8).to(F64)
    exp, man = mag // 2, (mag % 2).to(F64)
    val = torch.where(exp == 0, 0.5 * man, torch.exp2((exp - 1).to(F64)) * (1.0 + 0.5 * man)) * sign
    del nib, mag, sign, exp, man
    c = s["codes"].to(torch.int64)
    ce, cm = c // 8, (c % 8).to(F64)
    scale = torch.where(ce == 0, cm * 2.0 ** -9, torch.exp2((ce - 7).to(F64)) * (1.0 + cm / 8.0)) * s["sg"].to(F64)
    return (val.reshape(m, n // 16, 16) * scale[:, :, None]).reshape(m, n)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "checkpoint":
        return {"x": _exact_checkpoint(s["x"], case["format"])}
    w, ids = _weight64(s), s["ids"]
    if case["kind"] == "project":
        x = s["x"].to(F64)
        y = x @ w.T
        for a in ids.unique().tolist():
            if a >= 0:
                rows = (ids == a).nonzero().squeeze(1)
                low = x[rows] @ s["a"][a].to(F64).T
                y[rows] += s["alpha"][a].to(F64) * (low @ s["b"][a].to(F64).T)
        return {"y": y}
    x, dy = _load(s["q"], s["scales"], case["format"], F64), s["dy"].to(F64)
    dx = dy @ w
    da, db = torch.zeros_like(s["a"], dtype=F64), torch.zeros_like(s["b"], dtype=F64)
    for a in ids.unique().tolist():
        if a >= 0:
            rows = (ids == a).nonzero().squeeze(1)
            al, wa, wb = s["alpha"][a].to(F64), s["a"][a].to(F64), s["b"][a].to(F64)
            back = al * (dy[rows] @ wb)
            dx[rows] += back @ wa
            da[a] = back.T @ x[rows]
            db[a] = al * (dy[rows].T @ (x[rows] @ wa.T))
    return {"dx": dx, "da": da, "db": db}
