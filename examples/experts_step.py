"""A mixture-of-experts layer quantized to NVFP4, its router trained and served: the calls of this library in the order
a program makes them.

1. Quantization: each expert's matrices, with h = diag(X^T X) over the tokens that calibrate them.
2. Training steps of the router before the frozen packed experts, against the unquantized layer's outputs: the router's
   scores, the choice of experts, the layer; its gradients back to the scores and to x; both clipped by their global norm.
3. Serving: one decoding batch.

    python examples/experts_step.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_28113_gb300 as hs  # noqa: E402
from paper_2608_28113_gb300 import workloads as wl  # noqa: E402


def quantize(weights: torch.Tensor, x: torch.Tensor, window: int = 4):
    """(packed, codes, scale) of weights [experts, m, n] under the activations x [tokens, n]."""
    count, m, n = weights.shape
    h = torch.zeros(n, dtype=torch.float32, device=x.device)
    hs.hscale_hessian_diag_accumulate(x, h)
    packed = torch.empty(count, m, n // 2, dtype=torch.uint8, device=x.device)
    codes = torch.empty(count, m, n // 16, dtype=torch.uint8, device=x.device)
    scale = torch.empty(count, dtype=torch.float32, device=x.device)
    workspace = torch.empty(hs.hscale_rtn_workspace_bytes(), dtype=torch.uint8, device=x.device)
    sg = torch.empty(1, dtype=torch.float32, device=x.device)
    for e in range(count):
        hs.hscale_rtn_scales(weights[e], sg, codes[e], workspace)
        hs.hscale_refine_scales(weights[e], h, sg, codes[e].clone(), window, window, codes[e], packed[e])
        scale[e:e + 1] = sg
    return packed, codes, scale


def run(n: int = 512, inner: int = 256, experts: int = 16, k: int = 4, tokens: int = 1024, steps: int = 20, rate: float = 1e-2,
        max_norm: float = 1.0, seed: int = 0, device: str = "cuda"):
    """Losses (mean squared error to the unquantized layer under another router), gradient norms, and the served outputs."""
    make = lambda m, c, s: torch.stack([wl.weight(m, c, 0.05, seed + 10 * s + e) for e in range(experts)]).to(device)  # noqa: E731
    gate, up, down = make(inner, n, 1), make(inner, n, 2), make(n, inner, 3)
    x = wl.activation_chunk(tokens, wl.channel_magnitudes(n, 0.5, 4, 8.0, seed), seed, 0).to(device)
    inside = (torch.nn.functional.silu(x.float() @ gate[0].float().T) * (x.float() @ up[0].float().T)).to(torch.bfloat16)
    packed = quantize(gate, x), quantize(up, x), quantize(down, inside)

    g = torch.Generator(device=device).manual_seed(seed)
    teacher, router = (torch.randn(experts, n, generator=g, device=device) / n ** 0.5 for _ in range(2))
    ids = torch.empty(tokens, k, dtype=torch.int32, device=device)
    weights = torch.empty(tokens, k, dtype=torch.float32, device=device)

    def target():
        hs.hscale_route(x.float() @ teacher.T, ids, weights, True)
        out = torch.zeros(tokens, n, device=device)
        for e in range(experts):
            share = ((ids == e) * weights).sum(1, keepdim=True)
            h = torch.nn.functional.silu(x.float() @ gate[e].float().T) * (x.float() @ up[e].float().T)
            out += share * (h @ down[e].float().T)
        return out

    want = target()
    y, dx = torch.empty(tokens, n, dtype=torch.bfloat16, device=device), torch.empty(tokens, n, dtype=torch.bfloat16, device=device)
    dweights, norm = torch.empty_like(weights), torch.empty(1, device=device)
    nbytes = hs.hscale_experts_backward_workspace_bytes(tokens, k, n, inner, experts)
    nbytes = max(nbytes, hs.hscale_experts_workspace_bytes(tokens, k, n, inner, experts))
    workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    losses, norms = [], []
    for _ in range(steps):
        logits = x.float() @ router.T
        hs.hscale_route(logits, ids, weights, True)
        hs.hscale_experts(x, ids, weights, *packed, hs.HSCALE_ACT_SILU, y, workspace)
        error = y.float() - want
        losses.append((error * error).mean())
        dy = (error * (2.0 / error.numel())).to(torch.bfloat16)
        hs.hscale_experts_backward(dy, x, ids, weights, *packed, hs.HSCALE_ACT_SILU, dx, dweights, workspace)
        dlogits = torch.empty_like(logits)
        hs.hscale_route_backward(None, ids, weights, dweights, True, dlogits)
        drouter = dlogits.T @ x.float()
        hs.hscale_grad_clip([drouter, dx], max_norm, norm)
        norms.append(norm.clone())
        router -= rate * drouter / (drouter.norm() + 1e-12)

    batch = x[:5]
    few_ids, few_weights = ids[:5].clone(), weights[:5].clone()
    hs.hscale_route(batch.float() @ router.T, few_ids, few_weights, True)
    served = torch.empty(5, n, dtype=torch.bfloat16, device=device)
    hs.hscale_experts(batch, few_ids, few_weights, *packed, hs.HSCALE_ACT_SILU, served)
    return [v.item() for v in losses], [v.item() for v in norms], served


if __name__ == "__main__":
    losses, norms, served = run()
    print(f"mean squared error to the unquantized layer: {losses[0]:.3e}, {losses[-1]:.3e} after {len(losses) - 1} steps of the router")
    print(f"gradient norm {norms[0]:.3e}, {norms[-1]:.3e}; served a batch of {served.shape[0]} tokens")
