"""The mixture-of-experts operators' and the gradient norm's refusals, on the CPU: nothing is enqueued for a bad
argument.  And the tests' own 64-bit gradients, by differences."""
import ctypes

import pytest
import torch

import paper_2608_28113_gb300 as hs
from expert_reference import dequantized, experts, experts_backward
from paper_2608_28113_gb300 import build

OK, ERR_NULL, ERR_SHAPE, ERR_ALIGN, ERR_ARG, ERR_CUDA, ERR_WS = range(7)
P = 4096  # an aligned address that no refused call touches


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hs.load()


ROUTE = dict(logits=P, type=0, tokens=4, experts=16, ld=16, k=2, renormalize=1, ids=P, weights=P, stream=None)
ROUTING = [(dict(tokens=-1), ERR_SHAPE), (dict(experts=0), ERR_SHAPE), (dict(experts=1025, ld=1025, ld_out=1025), ERR_SHAPE),
           (dict(k=0), ERR_SHAPE), (dict(k=33), ERR_SHAPE), (dict(tokens=1 << 31), ERR_SHAPE), (dict(type=2), ERR_ARG),
           (dict(ids=None), ERR_NULL), (dict(weights=None), ERR_NULL), (dict(ids=P + 2), ERR_ALIGN), (dict(weights=P + 2), ERR_ALIGN)]


@pytest.mark.parametrize("change, status", ROUTING + [
    (dict(ld=15), ERR_SHAPE), (dict(logits=None), ERR_NULL), (dict(logits=P + 1), ERR_ALIGN), (dict(type=1, logits=P + 2), ERR_ALIGN),
    (dict(ld=1 << 62), ERR_SHAPE), (dict(tokens=0, logits=None, ids=None, weights=None), OK)])
def test_route_refusals(lib, change, status):
    assert lib.hscale_route(*{**ROUTE, **{k: v for k, v in change.items() if k in ROUTE}}.values()) == status


BACK = dict(logits=P, type=0, tokens=4, experts=16, ld=16, ids=P, weights=P, dweights=P, k=2, renormalize=0, out=P, ld_out=16,
            stream=None)


@pytest.mark.parametrize("change, status", ROUTING + [
    (dict(ld=15), ERR_SHAPE), (dict(ld_out=15), ERR_SHAPE), (dict(logits=None), ERR_NULL), (dict(dweights=None), ERR_NULL),
    (dict(out=None), ERR_NULL), (dict(out=P + 1), ERR_ALIGN), (dict(dweights=P + 1), ERR_ALIGN),
    (dict(renormalize=1, logits=None, out=None), ERR_NULL), (dict(tokens=0, logits=None, out=None, ids=None), OK)])
def test_route_backward_refusals(lib, change, status):
    assert lib.hscale_route_backward(*{**BACK, **{k: v for k, v in change.items() if k in BACK}}.values()) == status


WEIGHTS = {f"{m}_{part}": P for m in ("gate", "up", "down") for part in ("packed", "codes", "scale")}
EXPERTS = dict(x=P, tokens=4, n=64, ld_x=64, ids=P, weights=P, k=2, **WEIGHTS, experts=16, inner=32, act=0, y=P, ld_y=64, ws=P,
               ws_bytes=1 << 30, stream=None)
LAYER = [(dict(tokens=-1), ERR_SHAPE), (dict(n=72, ld_x=72, ld_y=72, ld_dy=72, ld_dx=72), ERR_SHAPE), (dict(inner=40), ERR_SHAPE),
         (dict(inner=-16), ERR_SHAPE), (dict(experts=0), ERR_SHAPE), (dict(experts=1025), ERR_SHAPE), (dict(k=0), ERR_SHAPE),
         (dict(k=33), ERR_SHAPE), (dict(act=2), ERR_ARG), (dict(act=-1), ERR_ARG), (dict(ids=None), ERR_NULL),
         (dict(weights=None), ERR_NULL), (dict(ids=P + 1), ERR_ALIGN), (dict(weights=P + 2), ERR_ALIGN), (dict(x=None), ERR_NULL),
         (dict(x=P + 8), ERR_ALIGN), (dict(ld_x=56), ERR_SHAPE), (dict(ld_x=68), ERR_ALIGN), (dict(ws=None), ERR_WS),
         (dict(ws_bytes=255), ERR_WS), (dict(ws=P + 16), ERR_WS), (dict(tokens=1 << 26, n=1 << 30, ld_x=1 << 30), ERR_SHAPE)]
# slots times inner, the weights, and the tiles' blocks past what the kernels count
WIDE = dict(ld_x=1 << 24, ld_y=1 << 24, ld_dy=1 << 24, ld_dx=1 << 24, ws_bytes=(1 << 64) - 1)
LAYER += [(dict(tokens=(1 << 26) - 1, k=32, inner=1 << 30, **WIDE), ERR_SHAPE), (dict(n=1 << 24, inner=1 << 24, experts=1024, **WIDE), ERR_SHAPE),
          (dict(tokens=1 << 16, k=1, n=1 << 20, inner=1 << 20, experts=1, **WIDE), ERR_SHAPE)]
LAYER += [({name: None}, ERR_NULL) for name in WEIGHTS]
LAYER += [({f"{m}_packed": P + 4}, ERR_ALIGN) for m in ("gate", "up", "down")]
LAYER += [({f"{m}_scale": P + 2}, ERR_ALIGN) for m in ("gate", "up", "down")]


@pytest.mark.parametrize("change, status", LAYER + [
    (dict(y=None), ERR_NULL), (dict(y=P + 2), ERR_ALIGN), (dict(ld_y=56), ERR_SHAPE), (dict(ld_y=68), ERR_ALIGN),
    (dict(tokens=0, x=None, y=None, ids=None, ws=None), OK), (dict(n=0, x=None, y=None, ws=None), OK)])
def test_experts_refusals(lib, change, status):
    assert lib.hscale_experts(*{**EXPERTS, **{k: v for k, v in change.items() if k in EXPERTS}}.values()) == status


EXPERTS_BACK = dict(dy=P, tokens=4, n=64, ld_dy=64, x=P, ld_x=64, ids=P, weights=P, k=2, **WEIGHTS, experts=16, inner=32, act=0, dx=P,
                    ld_dx=64, dweights=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change, status", LAYER + [
    (dict(dy=None), ERR_NULL), (dict(dy=P + 2), ERR_ALIGN), (dict(ld_dy=56), ERR_SHAPE), (dict(dx=P + 2), ERR_ALIGN),
    (dict(ld_dx=56), ERR_SHAPE), (dict(dweights=P + 2), ERR_ALIGN), (dict(dx=None, dweights=None), OK),
    (dict(tokens=0, x=None, dy=None, dx=None, ws=None), OK)])
def test_experts_backward_refusals(lib, change, status):
    assert lib.hscale_experts_backward(*{**EXPERTS_BACK, **{k: v for k, v in change.items() if k in EXPERTS_BACK}}.values()) == status


def test_workspace_queries(lib):
    for f in (hs.hscale_experts_workspace_bytes, hs.hscale_experts_backward_workspace_bytes):
        assert f(0, 2, 64, 64, 4) == 0 and f(4, 2, 0, 64, 4) == 0 and f(4, 2, 64, 0, 4) == 0
        assert f(4, 2, 64, 32, 4) > 0
        assert f(4096, 8, 4096, 2048, 64) >= f(4096, 8, 4096, 2048, 1) - 4096 * 8
        assert f(1 << 26, 32, 1 << 14, 1 << 14, 64) > 1 << 46  # no overflow into a small number
        assert f((1 << 26) - 1, 32, 16, 1 << 30, 64) > 1 << 46 and f(1 << 62, 32, 64, 64, 4) > 1 << 46
    # what a call of fewer tokens needs is no more
    sizes = [hs.hscale_experts_workspace_bytes(t, 8, 512, 256, 64) for t in range(1, 300)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_grad_refusals(lib):
    def call(count=2, tensors=(P, P), sizes=(8, 8), types=(0, 1), max_norm=1.0, norm=P, out=None, ws=P, nbytes=1 << 20):
        array = lambda kind, v: None if v is None else (kind * len(v))(*v)  # noqa: E731
        args = (array(ctypes.c_void_p, tensors), array(ctypes.c_int64, sizes), array(ctypes.c_int32, types), count)
        return lib.hscale_grad_clip(*args, max_norm, norm, array(ctypes.c_void_p, out), ws, nbytes, None)

    assert call(count=-1) == ERR_SHAPE
    assert call(sizes=(8, -1)) == ERR_SHAPE
    assert call(sizes=(8, 1 << 60)) == ERR_SHAPE
    assert call(types=(0, 3)) == ERR_ARG
    assert call(max_norm=-1.0) == ERR_ARG and call(max_norm=float("nan")) == ERR_ARG
    assert call(norm=None) == ERR_NULL and call(tensors=None) == ERR_NULL and call(sizes=None) == ERR_NULL
    assert call(tensors=(P, None)) == ERR_NULL and call(out=(P, None)) == ERR_NULL
    assert call(tensors=(P + 1, P)) == ERR_ALIGN and call(tensors=(P, P + 2)) == ERR_ALIGN and call(out=(P, P + 2)) == ERR_ALIGN
    assert call(norm=P + 2) == ERR_ALIGN
    assert call(ws=None) == ERR_WS and call(nbytes=16) == ERR_WS and call(ws=P + 16) == ERR_WS


def test_binding_refuses_what_it_cannot_marshal(lib):
    f, ids = torch.zeros(2, 8), torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(TypeError):
        hs.hscale_route(f, ids, torch.zeros(2, 2), True)
    with pytest.raises(TypeError):
        hs.hscale_tensors([f])
    with pytest.raises(TypeError):
        hs.hscale_grad_norm([], torch.zeros(1))
    x = torch.zeros(2, 32, dtype=torch.bfloat16)
    with pytest.raises((TypeError, ValueError)):
        hs.hscale_experts(x, ids, torch.zeros(2, 2), (None,) * 3, (None,) * 3, (None,) * 3, 0, x)


@pytest.mark.parametrize("kind", [0, 1])
def test_reference_gradients_by_differences(kind):
    g = torch.Generator().manual_seed(kind)
    t, n, inner, count, k = 3, 16, 16, 3, 2

    def matrix(rows, cols):
        return (torch.randint(256, (count, rows, cols // 2), generator=g).to(torch.uint8),
                torch.randint(50, 60, (count, rows, cols // 16), generator=g).to(torch.uint8), torch.rand(count, generator=g) * 0.2)

    weights = matrix(inner, n), matrix(inner, n), matrix(n, inner)
    dense = [tuple(dequantized(m, e) for m in weights) for e in range(count)]
    x = torch.randn(t, n, generator=g, dtype=torch.float64)
    dy = torch.randn(t, n, generator=g, dtype=torch.float64)
    ids = torch.tensor([[0, 2], [1, 1], [2, -1]], dtype=torch.int32)
    w = torch.rand(t, k, generator=g, dtype=torch.float64)
    dx, _, dw, _ = experts_backward(dy, x, ids, w, *weights, kind)

    def loss(x, w):
        return (experts(x, ids, w, *weights, kind, w=dense)[0] * dy).sum().item()

    step = 1e-5
    for value, grad, f in ((x, dx, lambda v: loss(v, w)), (w, dw, lambda v: loss(x, v))):
        for i in range(value.numel()):
            hi, lo = value.clone(), value.clone()
            hi.view(-1)[i] += step
            lo.view(-1)[i] -= step
            slope = (f(hi) - f(lo)) / (2 * step)
            assert abs(slope - grad.view(-1)[i].item()) <= 1e-6 * (1 + abs(slope)) * 10
