"""Clipping by a factor that fp32 holds with few bits or not at all."""
import math

import pytest
import torch

import paper_2608_28113_gb300 as hs

pytestmark = pytest.mark.gpu
BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64


# (size of the elements, largest norm): factors of 1e-40, 1e-46 and 1e-73; just above and below fp32's least normal number; and
# results that are themselves below it
@pytest.mark.parametrize("scale, limit", [(1e36, 1e-2), (1e36, 1e-8), (1e36, 1e-35), (1e10, 7e-27), (1e10, 1e-26), (1e30, 1e-39),
                                          (1e36, 0.0)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("inplace", [False, True])
def test_factors_below_fp32s_range(scale, limit, dtype, inplace):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()
    g = torch.Generator().manual_seed(5)
    grads = [(torch.randn(n, generator=g, dtype=F64) * scale).to(kind).cuda()
             for n, kind in ((5000, dtype), (37, F32), (4097, dtype), (300, F16 if scale < 1e4 else BF16))]
    before = [t.clone() for t in grads]
    norm = torch.empty(1, device="cuda")
    out = None if inplace else [torch.empty_like(t) for t in grads]
    hs.hscale_grad_clip(grads, limit, norm, out)
    want = math.sqrt(sum((t.to(F64) ** 2).sum().item() for t in before))
    assert abs(norm.item() - want) <= want * 64 * 2.0 ** -24
    limit = torch.tensor(limit, dtype=F32).item()
    for b, o in zip(before, out or grads):
        exact = b.to(F64) * (limit / want)
        # the norm's 64 2^-24, the factor's and the product's roundings, the type's; at least half of its least number, and of
        # fp32's before that
        tol = exact.abs() * (torch.finfo(o.dtype).eps / 2 + 68 * 2.0 ** -24) + torch.finfo(o.dtype).tiny * torch.finfo(o.dtype).eps * 0.51
        assert ((o.to(F64) - exact).abs() <= tol + 2.0 ** -150).all()
