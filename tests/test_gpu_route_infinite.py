"""A logit of +Inf counts as its type's largest finite number, in every kernel of the router and in its gradient."""
import math

import pytest
import torch

import paper_2608_28113_gb300 as hs
from expert_reference import route, route_backward

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


def logits(experts, dtype):
    """Rows with +Inf and the type's largest number, in both orders, several of each, and beside ordinary ones."""
    largest = torch.finfo(dtype).max
    v = torch.randn(6, experts, generator=torch.Generator().manual_seed(experts))
    v[0, 1], v[0, experts - 1] = math.inf, largest
    v[1, 1], v[1, experts - 1] = largest, math.inf
    v[2, [0, 2, experts - 2]], v[2, 1] = math.inf, largest
    v[3, :] = largest
    v[3, experts // 2] = math.inf
    v[4, 3] = math.inf
    v[5, [0, experts - 1]] = largest
    return v.to(dtype)


@pytest.mark.parametrize("experts", [5, 32, 61, 128, 256, 257, 1024])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("renormalize", [False, True])
def test_infinite_logits(experts, dtype, renormalize):
    v, k = logits(experts, dtype), 4
    finite = v.clamp(max=torch.finfo(dtype).max)
    want_ids, want = route(finite, k, renormalize)
    ids, w = torch.empty(6, k, dtype=I32, device=DEV), torch.empty(6, k, device=DEV)
    hs.hscale_route(v.to(DEV), ids, w, renormalize)
    assert torch.equal(ids.cpu(), want_ids)
    # of equal numbers the weights are 1 / their number, of others exp(-1e38) = 0: a quotient and a sum of whole numbers
    assert ((w.cpu().double() - want).abs() <= want * 4 * 2.0 ** -24).all()

    dw = torch.randn(6, k, generator=torch.Generator().manual_seed(1)).to(DEV)
    out = torch.empty(6, experts, dtype=dtype, device=DEV)
    hs.hscale_route_backward(v.to(DEV), ids, w, dw, renormalize, out)
    back = route_backward(finite, ids.cpu(), w.cpu(), dw.cpu(), renormalize)
    # sums of at most four products below 4, and the type's rounding
    tol = back.abs() * torch.finfo(dtype).eps / 2 * 1.01 + dw.abs().max().item() * 16 * 2.0 ** -24
    assert ((out.cpu().double() - back).abs() <= tol).all()
