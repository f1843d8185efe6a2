"""The mixture-of-experts operators in plain 64-bit operations, for the tests."""
import math

import torch

F64 = torch.float64


def dequantized(weight, e):
    """Expert e's matrix of (packed, codes, scale)."""
    packed, codes, scale = (t.cpu() for t in weight)
    p = packed[e].to(torch.int64)
    nib = torch.stack((p % 16, p // 16), 2).reshape(p.shape[0], -1)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=F64)
    v = grid[nib % 8] * (1 - 2 * (nib // 8)).to(F64)
    c = (codes[e].to(torch.int64) % 128).clamp(1, 126)
    s = torch.where(c < 8, (c % 8).to(F64) * 2.0 ** -9, torch.exp2((c // 8 - 7).to(F64)) * (1 + (c % 8).to(F64) / 8))
    return v * s.repeat_interleave(16, 1) * scale[e].to(F64)


def activation(kind, g):
    """act(g) and act'(g): g s(q)."""
    c = 2 * math.sqrt(2 / math.pi)
    q = g if kind == 0 else c * (g + 0.044715 * g ** 3)
    dq = 1.0 if kind == 0 else c * (1 + 3 * 0.044715 * g ** 2)
    s = torch.sigmoid(q)
    return g * s, s + g * dq * s * torch.sigmoid(-q)


def experts(x, ids, weights, gate, up, down, kind, w=None):
    """y, and a bound of the kernels' error: both operands' roundings and the sums' (see `bound` below)."""
    t, k = ids.shape
    x, wt = x.to(F64), weights.to(F64)
    y, tol = torch.zeros_like(x), torch.zeros_like(x)
    for e in range(gate[0].shape[0]):
        rows, slot = (ids == e).nonzero(as_tuple=True)
        if rows.numel() == 0:
            continue
        gm, um, dm = w[e] if w else (dequantized(gate, e), dequantized(up, e), dequantized(down, e))
        g, u = x[rows] @ gm.T, x[rows] @ um.T
        a, _ = activation(kind, g)
        h, s = a * u, wt[rows, slot][:, None]
        # n products summed in fp32: n 2^-24 of the sum of magnitudes at most; |act'| < 1.13; the fast activation 2^-18;
        # h rounded to fp16 under a power of two of its 32 outputs, then of its row (the largest above 2^14): 2^-11 of it, or
        # twice half of fp16's least step, 2^-25 2^-14 of the row's largest
        dg, du = (x[rows].abs() @ m.abs().T * (x.shape[1] + 8) * 2.0 ** -24 for m in (gm, um))
        dh = (1.13 * dg + 2.0 ** -18 * a.abs()) * u.abs() + a.abs() * du + 2.0 ** -11 * h.abs() + 2.0 ** -38 * h.abs().amax(1, True)
        mag = (h.abs() + dh) @ dm.abs().T
        y.index_add_(0, rows, s * (h @ dm.T))
        tol.index_add_(0, rows, s.abs() * (dh @ dm.abs().T + mag * (dm.shape[1] + 8) * 2.0 ** -24))
    return y, tol + 2.0 ** -8 * (y.abs() + tol)


def experts_backward(dy, x, ids, weights, gate, up, down, kind):
    """dx, dweights and bounds of the kernels' errors."""
    x, dy, wt = x.to(F64), dy.to(F64), weights.to(F64)
    dx, tx = torch.zeros_like(x), torch.zeros_like(x)
    dw, tw = torch.zeros_like(wt), torch.zeros_like(wt)
    for e in range(gate[0].shape[0]):
        rows, slot = (ids == e).nonzero(as_tuple=True)
        if rows.numel() == 0:
            continue
        gm, um, dm = dequantized(gate, e), dequantized(up, e), dequantized(down, e)
        xe, s = x[rows], wt[rows, slot][:, None]
        g, u, dh = xe @ gm.T, xe @ um.T, dy[rows] @ dm
        a, slope = activation(kind, g)
        eps = 2.0 ** -24
        n, inner = x.shape[1], gm.shape[0]
        dg_, du_ = (xe.abs() @ m.abs().T * (n + 8) * eps for m in (gm, um))
        ddh = dy[rows].abs() @ dm.abs() * (n + 8) * eps
        # |act'| < 1.13 and |act''| < 1.1 for both activations; the activation's own error a few 2^-24
        ea, es = 1.13 * dg_ + 8 * eps * (a.abs() + 1), 1.1 * dg_ + 8 * eps
        dw[rows, slot] = (a * u * dh).sum(1)
        mags = (a.abs() + ea) * (u.abs() + du_) * (dh.abs() + ddh)
        tw[rows, slot] = ((ea * u.abs() + a.abs() * du_) * dh.abs() + (a * u).abs() * ddh).sum(1) * 1.01 + \
            mags.sum(1) * (inner / 32 + 40) * eps
        fg, fu = s * dh * u * slope, s * dh * a
        # the factors are rounded as h is, both under one power of two
        most = 2.0 ** -38 * torch.maximum(fg.abs(), fu.abs()).amax(1, True)
        eg = s.abs() * (ddh * (u * slope).abs() + dh.abs() * (du_ * slope.abs() + u.abs() * es)) * 1.01 + 2.0 ** -11 * fg.abs() + most
        eu = s.abs() * (ddh * a.abs() + dh.abs() * ea) * 1.01 + 2.0 ** -11 * fu.abs() + most
        dx.index_add_(0, rows, fg @ gm + fu @ um)
        err = eg @ gm.abs() + eu @ um.abs() + (fg.abs() @ gm.abs() + fu.abs() @ um.abs()) * (2 * inner + 8) * eps
        tx.index_add_(0, rows, err)
    return dx, tx + 2.0 ** -8 * (dx.abs() + tx), dw, tw


def route(logits, k, renormalize):
    v = logits.to(F64).cpu()
    v = torch.where(torch.isnan(v), -math.inf, v).clamp(max=torch.finfo(torch.float32).max)
    t, e = v.shape
    ids, weights = torch.full((t, k), -1, dtype=torch.int32), torch.zeros(t, k, dtype=F64)
    for i in range(t):
        order = sorted((j for j in range(e) if v[i, j] > -math.inf), key=lambda j: (-v[i, j].item(), j))[:k]
        if not order:
            continue
        p = torch.exp(v[i] - v[i].max())
        total = p[order].sum() if renormalize else p.sum()
        ids[i, :len(order)] = torch.tensor(order, dtype=torch.int32)
        weights[i, :len(order)] = p[order] / total
    return ids, weights


def route_backward(logits, ids, weights, dweights, renormalize):
    v = logits.to(F64).cpu()
    v = torch.where(torch.isnan(v), -math.inf, v).clamp(max=torch.finfo(torch.float32).max)
    t, e = v.shape
    out = torch.zeros(t, e, dtype=F64)
    for i in range(t):
        on = [j for j in range(ids.shape[1]) if 0 <= ids[i, j] < e]
        mean = sum(weights[i, j].item() * dweights[i, j].item() for j in on)
        if not renormalize and (v[i] > -math.inf).any():
            p = torch.exp(v[i] - v[i].max())
            p /= p.sum()
            out[i] = -p * mean
        for j in on:
            c = int(ids[i, j])
            out[i, c] += weights[i, j].item() * (dweights[i, j].item() - mean) if renormalize else p[c] * dweights[i, j].item()
    return out
