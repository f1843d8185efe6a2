"""The router and its gradient against plain 64-bit operations."""
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


def logits_of(t, e, dtype, pad, seed, kind="plain"):
    g = torch.Generator().manual_seed(seed)
    v = 2 * torch.randn(t, e, generator=g)
    if kind == "ties":
        v = torch.randint(-1, 2, (t, e), generator=g).float()
        v[0] = 0.0
        v[1, ::2] = -0.0
    if kind == "masked":
        v[:, torch.rand(e, generator=g) < 0.3] = -math.inf
        v[::5] = -math.inf  # rows without an expert
        v[torch.rand(t, e, generator=g) < 0.1] = math.nan
        v[3::7, e // 2] = math.inf
        v[4::9] = torch.finfo(dtype).min  # the lowest number is a number
    full = torch.full((t, e + pad), 7.0, dtype=dtype, device=DEV)
    full[:, :e] = v.to(dtype)
    return full[:, :e], full


SIZES = [(1, 1, 1), (1, 8, 8), (5, 3, 5), (3, 64, 8), (130, 61, 3), (17, 128, 8), (33, 200, 32), (9, 257, 6), (4, 1024, 16)]


def run(v, k, renormalize, stream=None):
    t = v.shape[0]
    ids, w = torch.full((t, k), 99, dtype=I32, device=DEV), torch.full((t, k), math.nan, device=DEV)
    hs.hscale_route(v, ids, w, renormalize, stream=stream)
    return ids, w


@pytest.mark.parametrize("t, e, k", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["plain", "ties", "masked"])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route(t, e, k, dtype, kind, renormalize):
    if t < 2 and kind == "ties":
        t = 2
    v, _ = logits_of(t, e, dtype, 3, t * e + k, kind)
    ids, w = run(v, k, renormalize)
    want_ids, want = route(v, k, renormalize)
    assert torch.equal(ids.cpu(), want_ids)
    # exp and the quotient a few units, a sum of e positive numbers at most (32 + e / 32) roundings, and the difference
    # l - max, exact to 2^-24 of it, in the exponent
    span = torch.where(want > 0, -torch.log(want.clamp(min=1e-40)), 0.0).max().item() + 16
    assert ((w.cpu().double() - want).abs() <= want * (40 + span) * 2.0 ** -23 + 1e-38).all()
    again = run(v, k, renormalize)
    assert torch.equal(again[0], ids) and torch.equal(again[1], w)


@pytest.mark.parametrize("t, e, k", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["plain", "masked"])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route_backward(t, e, k, dtype, kind, renormalize):
    v, _ = logits_of(t, e, dtype, 5, 3 * t + e, kind)
    ids, w = run(v, k, renormalize)
    g = torch.Generator().manual_seed(1)
    dw = torch.randn(t, k, generator=g).to(DEV)
    dw[ids < 0] = math.nan  # of a choice that is none
    w[ids < 0] = math.nan
    full = torch.full((t, e + 9), 5.0, dtype=dtype, device=DEV)
    out = full[:, :e]
    hs.hscale_route_backward(None if renormalize else v, ids, w, dw, renormalize, out)
    want = route_backward(v, ids.cpu(), w.cpu(), dw.cpu(), renormalize)
    # magnitudes at most max |dw| (1 + k) of each p; roundings as above, then the type's
    size = dw[ids >= 0].abs().max().item() * 2 if (ids >= 0).any() else 0.0
    tol = want.abs() * torch.finfo(dtype).eps / 2 * 1.01 + size * 64 * 2.0 ** -23
    assert ((out.cpu().double() - want).abs() <= tol).all()
    assert (full[:, e:] == 5.0).all()


def test_differences():
    """The gradient is that of the weights, by central differences of the forward pass in 64 bits."""
    g = torch.Generator().manual_seed(4)
    v = torch.randn(4, 9, generator=g, dtype=torch.float64)
    dw = torch.randn(4, 3, generator=g)
    for renormalize in (False, True):
        ids, w = run(v.float().to(DEV), 3, renormalize)
        out = torch.empty(4, 9, device=DEV)
        hs.hscale_route_backward(v.float().to(DEV), ids, w, dw.to(DEV), renormalize, out)
        step = 1e-5
        for e in range(9):
            hi, lo = v.float().double(), v.float().double()
            hi[:, e] += step
            lo[:, e] -= step
            slope = ((route(hi, 3, renormalize)[1] - route(lo, 3, renormalize)[1]) * dw).sum(1) / (2 * step)
            assert ((out[:, e].cpu() - slope).abs() <= 1e-5).all()  # 2^-23 of sums below 8, and step^2


@pytest.mark.parametrize("renormalize", [False, True])
def test_an_expert_twice(renormalize):
    v = torch.randn(2, 6, device=DEV)
    ids = torch.tensor([[2, 2, 5], [1, 9, 1]], dtype=I32, device=DEV)
    w, dw = torch.rand(2, 3, device=DEV), torch.randn(2, 3, device=DEV)
    out = torch.empty(2, 6, device=DEV)
    hs.hscale_route_backward(v, ids, w, dw, renormalize, out)
    want = route_backward(v, ids.cpu(), w.cpu(), dw.cpu(), renormalize)
    assert ((out.cpu() - want).abs() <= 1e-5).all()


def test_streams_and_graphs():
    v, _ = logits_of(64, 64, BF16, 0, 9)
    want = run(v, 4, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(v, 4, True, stream=side)
    side.synchronize()
    ids, w = torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hs.hscale_route(v, ids, w, True)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(want, got, (ids, w)):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_no_tokens():
    v = torch.empty(0, 8, device=DEV)
    ids, w = run(v, 2, True)
    hs.hscale_route_backward(v, ids, w, w, False, torch.empty(0, 8, device=DEV))
