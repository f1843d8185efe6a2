"""The gradients' norm and clipping against plain 64-bit operations."""
import math

import pytest
import torch

import paper_2608_28113_gb300 as hs

pytestmark = pytest.mark.gpu
BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


def tensors(sizes, dtypes, scale=1.0, seed=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        dtype = dtypes[i % len(dtypes)]
        room = torch.empty(n + shift, dtype=dtype, device=DEV)
        room[shift:] = (torch.randn(n, generator=g) * scale).to(dtype)
        out.append(room[shift:])
    return out


def norm_of(parts):
    return math.sqrt(sum((t.to(F64) ** 2).sum().item() for t in parts))


# fp32 sums of at most some dozens of squares a thread, then fp64
NORM_TOL = 64 * 2.0 ** -24

SIZES = [[1], [7], [16], [4096], [4097], [0, 5, 0], [1, 2, 3, 1000, 0, 65536 + 3], [12345] * 64, [33] * 65, [100] * 1000,
         [5] * 2311, [3 << 20]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("dtypes", [[BF16], [F32], [F16, F32, BF16]])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_and_clip(sizes, dtypes, shift):
    grads = tensors(sizes, dtypes, seed=len(sizes), shift=shift)
    want = norm_of(grads)
    norm = torch.full((1,), -1.0, device=DEV)
    hs.hscale_grad_norm(grads, norm)
    assert abs(norm.item() - want) <= want * NORM_TOL
    for limit in (0.5 * want, 2.0 * want + 1.0):
        out = [torch.full_like(t, 9.0) for t in grads]
        before = [t.clone() for t in grads]
        hs.hscale_grad_clip(grads, limit, norm, out)
        assert abs(norm.item() - want) <= want * NORM_TOL
        factor = min(1.0, limit / want) if want > 0 else 1.0
        for t, b, o in zip(grads, before, out):
            assert torch.equal(t, b)
            if factor == 1.0:
                assert torch.equal(o, t)
            else:
                exact = t.to(F64) * factor
                # the factor, the product and the rounding to the type
                tol = exact.abs() * (torch.finfo(t.dtype).eps / 2 + 2 * NORM_TOL) + torch.finfo(t.dtype).tiny * torch.finfo(t.dtype).eps
                assert ((o.to(F64) - exact).abs() <= tol).all()
        inplace = [b.clone() for b in before]
        hs.hscale_grad_clip(inplace, limit, norm)
        assert all(torch.equal(a, b) for a, b in zip(inplace, out))


@pytest.mark.parametrize("scale", [1e-40, 1e-30, 1e-22, 1e-15, 1e10, 1e18, 1e30, 1e37])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norms_whose_squares_leave_the_range(scale, dtype):
    g = torch.Generator().manual_seed(3)
    grads = [(torch.rand(5000, generator=g, dtype=F64) * scale).to(dtype).to(DEV), torch.zeros(70, dtype=dtype, device=DEV)]
    norm = torch.empty(1, device=DEV)
    hs.hscale_grad_norm(grads, norm)
    want = norm_of(grads)
    if want > torch.finfo(F32).max * (1 + 2.0 ** -25):  # 4.03e38, at 1e37: the norm, an fp32 number, rounds to Inf
        assert norm.item() == math.inf
    else:
        assert abs(norm.item() - want) <= want * NORM_TOL + 2.0 ** -149


def test_large_and_small_together():
    a = torch.full((64,), 3e25, device=DEV)
    b = torch.full((1000,), 1e-30, device=DEV)
    norm = torch.empty(1, device=DEV)
    hs.hscale_grad_norm([b, a, b], norm)
    assert abs(norm.item() - 8 * 3e25) <= 8 * 3e25 * NORM_TOL


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_what_is_not_finite_scales_nothing(value):
    grads = tensors([100, 5000], [F32, BF16])
    grads[1][4321] = value
    before = [t.clone() for t in grads]
    norm = torch.empty(1, device=DEV)
    hs.hscale_grad_clip(grads, 1e-3, norm)
    assert not math.isfinite(norm.item()) and math.isnan(norm.item()) == math.isnan(value)
    for a, b in zip(grads, before):
        assert torch.equal(a.nan_to_num(1.0), b.nan_to_num(1.0))


def test_limits():
    grads = tensors([50], [F32])
    norm = torch.empty(1, device=DEV)
    before = grads[0].clone()
    hs.hscale_grad_clip(grads, math.inf, norm)
    assert torch.equal(grads[0], before)
    hs.hscale_grad_clip(grads, 0.0, norm)
    assert (grads[0] == 0).all()
    hs.hscale_grad_clip(grads, 0.0, norm)
    assert norm.item() == 0 and (grads[0] == 0).all()
    hs.hscale_grad_norm([], norm.fill_(5.0))
    assert norm.item() == 0
    hs.hscale_grad_clip([torch.empty(0, device=DEV)], 1.0, norm.fill_(5.0))
    assert norm.item() == 0


def test_lists_streams_and_graphs():
    grads = tensors([4096 * 3 + 5, 999, 12, 70000] * 300, [BF16, F32], seed=5)
    held = hs.hscale_tensors(grads)
    assert hs.hscale_tensors(held) is held
    norm, out = torch.empty(1, device=DEV), [torch.empty_like(t) for t in grads]
    hs.hscale_grad_clip(held, 1.0, norm, out)
    want, first = norm.item(), [t.clone() for t in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    hs.hscale_grad_clip(held, 1.0, norm.fill_(0), out, stream=side)
    side.synchronize()
    assert norm.item() == want and all(torch.equal(a, b) for a, b in zip(out, first))
    for t in out:
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hs.hscale_grad_clip(held, 1.0, norm, out)
    norm.fill_(0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert norm.item() == want and all(torch.equal(a, b) for a, b in zip(out, first))


def test_refusals_on_the_gpu():
    a = torch.ones(8, device=DEV)
    norm = torch.empty(1, device=DEV)
    with pytest.raises(ValueError):
        hs.hscale_grad_clip([a, a], 1.0, norm)            # written twice
    with pytest.raises(ValueError):
        hs.hscale_grad_clip([a[:5], a[4:]], 1.0, norm)    # written by two
    with pytest.raises(ValueError):
        hs.hscale_grad_clip([a], 1.0, norm, [a.bfloat16()])
    with pytest.raises(ValueError):
        hs.hscale_grad_norm([a.view(2, 4).t()], norm)
    with pytest.raises(TypeError):
        hs.hscale_grad_norm([a.double()], norm)
    with pytest.raises(hs.HScaleError):
        hs.hscale_grad_clip([a], -1.0, norm)
    with pytest.raises(hs.HScaleError):
        hs.hscale_grad_clip([a], math.nan, norm)
    hs.hscale_grad_norm([a, a], norm)  # read twice is no harm
    assert abs(norm.item() - 4.0) < 1e-6
