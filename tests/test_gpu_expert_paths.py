"""The mixture-of-experts operators as programs meet them: router, layer, their gradients and clipping one after
another; rows and experts further than 2^32 bytes apart; the products' waits running out; the example."""
import importlib.util
import pathlib

import pytest
import torch

import paper_2608_28113_gb300 as hs
from expert_reference import activation, dequantized, experts, experts_backward
from test_gpu_experts import clean, layer, matrices, rows
from test_gpu_failure import both, starved  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
BF16, F32, F64, U8, I32 = torch.bfloat16, torch.float32, torch.float64, torch.uint8, torch.int32
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


def test_the_example_runs():
    path = pathlib.Path(__file__).resolve().parents[1] / "examples" / "experts_step.py"
    spec = importlib.util.spec_from_file_location("experts_step", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms, served = example.run(n=128, inner=64, experts=8, k=2, tokens=96, steps=3)
    assert len(losses) == len(norms) == 3
    assert all(v == v and v >= 0 for v in losses + norms)
    assert served.shape == (5, 128) and served.isfinite().all()


@pytest.mark.parametrize("t", [7, 150])
@pytest.mark.parametrize("renormalize", [False, True])
def test_router_layer_and_gradients_together(t, renormalize):
    """y = sum_j w_j(l) E_j(x) for router scores l: the gradients for l and x of the operators one after another, as they are
    used, against autograd's in 64 bits; then both clipped together."""
    n, inner, count, k = 128, 96, 6, 2
    g = torch.Generator().manual_seed(t)
    x, _ = rows(t, n, 0, g)
    gate, up, down = matrices(count, inner, n, g), matrices(count, inner, n, g), matrices(count, n, inner, g)
    logits = torch.randn(t, count, generator=g).to(DEV)
    dy, _ = rows(t, n, 0, g)
    ids, w = torch.empty(t, k, dtype=I32, device=DEV), torch.empty(t, k, device=DEV)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dw, dl = torch.empty_like(w), torch.empty_like(logits)
    hs.hscale_route(logits, ids, w, renormalize)
    hs.hscale_experts(x, ids, w, gate, up, down, 0, y)
    hs.hscale_experts_backward(dy, x, ids, w, gate, up, down, 0, dx, dw)
    hs.hscale_route_backward(logits, ids, w, dw, renormalize, dl)

    # the definition, differentiated by torch
    x64, l64 = x.cpu().double().requires_grad_(), logits.cpu().double().requires_grad_()
    chosen = ids.cpu().long()
    p = torch.softmax(l64, 1)
    w64 = p.gather(1, chosen)
    if renormalize:
        w64 = w64 / w64.sum(1, keepdim=True)
    total = torch.zeros(t, n, dtype=F64)
    for e in range(count):
        gm, um, dm = dequantized(gate, e), dequantized(up, e), dequantized(down, e)
        h = activation(0, x64 @ gm.T)[0] * (x64 @ um.T)
        total = total + ((chosen == e).double() * w64).sum(1, keepdim=True) * (h @ dm.T)
    total.backward(dy.cpu().double())
    want_y, tol_y = experts(x.cpu(), ids.cpu(), w.cpu(), gate, up, down, 0)
    assert torch.allclose(want_y, total.detach(), rtol=1e-5, atol=1e-5 * total.abs().max().item())  # w is fp32
    assert ((y.cpu().double() - total.detach()).abs() <= tol_y + 1e-6 * total.abs().max()).all()
    want_dx, tol_dx, _, tol_dw = experts_backward(dy.cpu(), x.cpu(), ids.cpu(), w.cpu(), gate, up, down, 0)
    assert ((dx.cpu().double() - x64.grad).abs() <= tol_dx + 1e-6 * x64.grad.abs().max()).all()
    # dl = w (dw - mean) or p (dw - mean): twice the largest error of dw, and fp32's of numbers as large as dw
    bound = 2 * tol_dw.max() + 64 * 2.0 ** -24 * dw.abs().max().item()
    assert ((dl.cpu().double() - l64.grad).abs() <= bound).all()

    norm = torch.empty(1, device=DEV)
    want = torch.sqrt((dx.double() ** 2).sum() + (dl.double() ** 2).sum()).item()
    before = dx.clone(), dl.clone()
    hs.hscale_grad_clip([dx, dl], 0.25 * want, norm)
    assert abs(norm.item() - want) <= 64 * 2.0 ** -24 * want
    for a, b in zip((dx, dl), before):
        exact = b.double() * 0.25
        assert ((a.double() - exact).abs() <= exact.abs() * (torch.finfo(a.dtype).eps / 2 + 2.0 ** -16)).all()


@pytest.mark.parametrize("t", [20, 70])
def test_rows_far_apart(t):
    """Rows 2^26 + 64 elements apart and more: the last ones begin past 2^32 bytes, from 64 rows on past 2^32 elements."""
    n, ld = 128, (1 << 28) + 64 if t < 64 else (1 << 26) + 64
    if torch.cuda.mem_get_info()[0] < 2.5 * t * ld:
        pytest.skip("not enough memory")
    x, ids, w, gate, up, down = layer(t, n, 96, 5, 2, seed=9)
    far = torch.empty(t * ld, dtype=BF16, device=DEV).view(t, ld)
    fx, fy, fdy, fdx = far[:, :n], far[:, n:2 * n], far[:, 256:256 + n], far[:, 384:384 + n]
    fx.copy_(x)
    fdy.copy_(x.roll(1, 0))
    dy = fdy.contiguous()
    y, dx, dw = torch.empty(t, n, dtype=BF16, device=DEV), torch.empty(t, n, dtype=BF16, device=DEV), torch.empty_like(w)
    fdw = torch.empty_like(w)
    hs.hscale_experts(x, ids, w, gate, up, down, 0, y)
    hs.hscale_experts(fx, ids, w, gate, up, down, 0, fy)
    hs.hscale_experts_backward(dy, x, ids, w, gate, up, down, 0, dx, dw)
    hs.hscale_experts_backward(fdy, fx, ids, w, gate, up, down, 0, fdx, fdw)
    assert torch.equal(fy.contiguous(), y) and torch.equal(fdx.contiguous(), dx) and torch.equal(fdw, dw)
    logits = far.view(torch.uint8).view(t, 2 * ld)[:, 4096:4096 + 64].view(torch.float32)
    logits.copy_(torch.randn(t, 16, device=DEV))
    near_ids, near_w = torch.empty(t, 3, dtype=I32, device=DEV), torch.empty(t, 3, device=DEV)
    far_ids, far_w = torch.empty_like(near_ids), torch.empty_like(near_w)
    hs.hscale_route(logits.contiguous(), near_ids, near_w, True)
    hs.hscale_route(logits, far_ids, far_w, True)
    assert torch.equal(near_ids, far_ids) and torch.equal(near_w, far_w)


@pytest.mark.parametrize("n, inner", [(4096, 4096), (4128, 4064), (4112, 4080)])
def test_experts_past_4_gib(n, inner):
    """The last experts' matrices begin more than 2^32 bytes into theirs."""
    count, t = 560, 3
    if torch.cuda.mem_get_info()[0] < 5 * count * n * inner:
        pytest.skip("not enough memory")
    g = torch.Generator(device=DEV).manual_seed(1)

    def big(r, c):
        packed = torch.randint(256, (count, r, c // 2), generator=g, device=DEV, dtype=U8)
        codes = torch.randint(40, 80, (count, r, c // 16), generator=g, device=DEV, dtype=U8)
        return packed, codes, torch.full((count,), 1e-3, device=DEV)

    assert count * n * inner // 2 > 1 << 32
    weights = big(inner, n), big(inner, n), big(n, inner)
    x, dy = (torch.randn(t, n, generator=g, device=DEV).to(BF16) for _ in range(2))
    ids = torch.tensor([[559, 2], [558, 559], [0, 557]], dtype=I32, device=DEV)
    w = torch.rand(t, 2, generator=g, device=DEV)
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    hs.hscale_experts(x, ids, w, *weights, 0, y)
    hs.hscale_experts_backward(dy, x, ids, w, *weights, 0, dx, dw)
    used = sorted(set(ids.flatten().tolist()))
    few = [tuple(part[used].contiguous() for part in m) for m in weights]
    few_ids = torch.tensor([[used.index(v) for v in r] for r in ids.tolist()], dtype=I32, device=DEV)
    near, near_dx, near_dw = torch.empty_like(y), torch.empty_like(dx), torch.empty_like(dw)
    hs.hscale_experts(x, few_ids, w, *few, 0, near)
    hs.hscale_experts_backward(dy, x, few_ids, w, *few, 0, near_dx, near_dw)
    assert torch.equal(y, near) and torch.equal(dx, near_dx) and torch.equal(dw, near_dw)
    want, tol = experts(x.cpu(), few_ids.cpu(), w.cpu(), *few, 0)
    assert ((y.cpu().double() - want).abs() <= tol).all()


@pytest.mark.parametrize("t", [6, 3000])
def test_layer_of_a_starved_block(starved, monkeypatch, t):  # noqa: F811
    """What a block whose epilogue gives up owed is NaN, in whole tokens or outputs; the rest is what it was."""
    args = layer(t, 512, 256, 8, 2, seed=12, none=0.0)

    def call():
        y = torch.zeros(t, 512, dtype=BF16, device=DEV)
        hs.hscale_experts(*args, 0, y)
        return y

    got, want = both(starved, monkeypatch, call)
    lost = got.isnan()
    assert lost.any() and not want.isnan().any()
    assert torch.equal(got[~lost], want[~lost])

    dy, _ = rows(t, 512, 0, torch.Generator().manual_seed(3))

    def back():
        dx, dw = torch.zeros(t, 512, dtype=BF16, device=DEV), torch.zeros(t, 2, device=DEV)
        hs.hscale_experts_backward(dy, *args, 0, dx, dw)
        return torch.cat((dx.float(), dw), 1)

    got, want = both(starved, monkeypatch, back)
    lost = got.isnan()
    assert lost.any() and not want.isnan().any()
    assert torch.equal(got[~lost], want[~lost])


def test_calls_of_other_sizes_in_one_workspace():
    """Calls one after another on a stream may share a workspace, whatever an earlier one left there."""
    sets = [layer(t, n, inner, count, k, seed=t) for t, n, inner, count, k in
            [(300, 256, 128, 4, 2), (3, 512, 64, 8, 8), (90, 128, 272, 3, 1), (1, 256, 256, 16, 4)]]
    ws = torch.full((64 << 20,), 255, dtype=U8, device=DEV)
    for x, ids, w, gate, up, down in sets + sets[::-1]:
        y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
        dy = x.roll(1, 0).contiguous()
        hs.hscale_experts(x, ids, w, gate, up, down, 0, y, ws)
        hs.hscale_experts_backward(dy, x, ids, w, gate, up, down, 0, dx, dw, ws)
        want, tol = experts(x.cpu(), ids.cpu(), clean(w), gate, up, down, 0)
        assert ((y.cpu().double() - want).abs() <= tol).all()
        want_dx, tol_dx, want_dw, tol_dw = experts_backward(dy.cpu(), x.cpu(), ids.cpu(), clean(w), gate, up, down, 0)
        assert ((dx.cpu().double() - want_dx).abs() <= tol_dx).all()
        assert ((dw.cpu().double() - want_dw).abs() <= tol_dw).all()
