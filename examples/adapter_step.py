"""A linear layer quantized to NVFP4, then adapted and served: the calls of this library in the order a program makes
them.

1. Calibration and quantization: h = diag(X^T X) over calibration tokens, RTN codes, the H-Scale search.
2. Training steps of one low-rank adapter beside the frozen packed weight, against the layer's bf16 weight: the
   activations are kept in 8 bits between the forward and the backward pass.
3. Serving: one decoding batch whose tokens belong to different adapters (the trained one, another, none).

    python examples/adapter_step.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_28113_gb300 as hs  # noqa: E402
from paper_2608_28113_gb300 import workloads as wl  # noqa: E402


def quantize(w: torch.Tensor, x: torch.Tensor, k: int = 4):
    """Packed nibbles, codes and global scale of w under the activations x."""
    m, n = w.shape
    h = torch.zeros(n, dtype=torch.float32, device=w.device)
    hs.hscale_hessian_diag_accumulate(x, h)
    sg = torch.empty(1, dtype=torch.float32, device=w.device)
    codes = torch.empty(m, n // 16, dtype=torch.uint8, device=w.device)
    packed = torch.empty(m, n // 2, dtype=torch.uint8, device=w.device)
    workspace = torch.empty(hs.hscale_rtn_workspace_bytes(), dtype=torch.uint8, device=w.device)
    hs.hscale_rtn_scales(w, sg, codes, workspace)
    hs.hscale_refine_scales(w, h, sg, codes, k, k, codes, packed)
    return packed, codes, sg


def run(m: int = 512, n: int = 1024, tokens: int = 2048, rank: int = 16, steps: int = 30, rate: float = 5e-4, seed: int = 0,
        device: str = "cuda"):
    """Losses of the training steps (mean squared error to the unquantized layer), and the served outputs.

    The rate is Adam's step for an element of A or B. B starts at zero and has to reach about (error of a weight) /
    (element of A x sqrt(rank)), some 6e-3 for weights of deviation 0.02: a dozen steps of 5e-4."""
    w = wl.weight(m, n, 0.02, seed).to(device)
    x = wl.activation_chunk(tokens, wl.channel_magnitudes(n, 0.5, 4, 8.0, seed), seed, 0).to(device)
    packed, codes, sg = quantize(w, x)
    target = (x.float() @ w.float().T)

    g = torch.Generator(device=device).manual_seed(seed)
    a = (torch.randn(2, rank, n, generator=g, device=device) / n ** 0.5).to(torch.bfloat16)
    b = torch.zeros(2, m, rank, dtype=torch.bfloat16, device=device)
    alpha = torch.ones(2, dtype=torch.float32, device=device)
    y = torch.empty(tokens, m, dtype=torch.bfloat16, device=device)
    da, db = torch.empty_like(a), torch.empty_like(b)
    held = torch.empty(tokens, n, dtype=torch.uint8, device=device)
    held_scales = torch.empty(tokens, (n + 31) // 32, dtype=torch.uint8, device=device)
    nbytes = hs.hscale_project_backward_workspace_bytes(tokens, m, n, 2, rank)
    workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    ids = torch.zeros(tokens, dtype=torch.int32, device=device)  # adapter 0 is trained
    master = [a.float(), b.float()]
    moments = [(torch.zeros_like(t), torch.zeros_like(t)) for t in master]
    losses = []
    for step in range(1, steps + 1):
        hs.hscale_project(x, packed, codes, sg, a, b, alpha, ids, y, workspace)
        hs.hscale_checkpoint_save(x, hs.HSCALE_CHECKPOINT_INT8, held, held_scales)
        error = y.float() - target
        losses.append((error * error).mean())
        dy = (error * (2.0 / error.numel())).to(torch.bfloat16)
        hs.hscale_project_backward(dy, held, held_scales, hs.HSCALE_CHECKPOINT_INT8, packed, codes, sg, a, b, alpha, ids, None,
                                   da, db, workspace)
        for t, grad, param, (first, second) in zip(master, (da, db), (a, b), moments):
            first.lerp_(grad.float(), 0.1)
            second.lerp_(grad.float() ** 2, 0.01)
            scale = (1 - 0.99 ** step) ** 0.5 / (1 - 0.9 ** step)
            t -= rate * scale * first / (second.sqrt() + 1e-12)
            param.copy_(t)

    batch = x[:5]
    who = torch.tensor([0, -1, 1, 0, -1], dtype=torch.int32, device=device)
    served = torch.empty(5, m, dtype=torch.bfloat16, device=device)
    hs.hscale_project(batch, packed, codes, sg, a, b, alpha, who, served)
    return [v.item() for v in losses], served


if __name__ == "__main__":
    losses, served = run()
    print(f"mean squared error to the unquantized layer: {losses[0]:.3e} quantized, {losses[-1]:.3e} after {len(losses) - 1} steps")
    print(f"served a batch of {served.shape[0]} tokens, {served.shape[1]} outputs each")
