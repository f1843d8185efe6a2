"""The experts' precision where it is hardest to keep: rows whose largest element is 2^27 to 2^36 times those that decide an
output, and dy far from 1."""
import pytest
import torch

import paper_2608_28113_gb300 as hs
from expert_reference import activation, dequantized, experts, experts_backward
from test_gpu_experts import backward, layer, matrices, rows, run

pytestmark = pytest.mark.gpu
BF16, U8, I32 = torch.bfloat16, torch.uint8, torch.int32
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


def zero_column(weight, col):
    """The weight with zeros in a column."""
    packed = weight[0].clone()
    packed[:, :, col // 2] &= 0xF0 if col % 2 == 0 else 0x0F
    return packed, weight[1], weight[2]


def zero_row(weight, row):
    packed = weight[0].clone()
    packed[:, row] = 0
    return packed, weight[1], weight[2]


def with_outlier(t, cols, at, low, high, g):
    """bf16 rows of numbers of 2^low to 2^high, and 1.5 in column `at`."""
    size = torch.exp2(low + (high - low) * torch.rand(t, cols, generator=g))
    v = size * (1 - 2 * torch.randint(2, (t, cols), generator=g).float())
    v[:, at] = 1.5
    return v.to(BF16).to(DEV)


def far_codes(weight, g, low=1, high=9):
    """The weight under codes of 2^-9 to 2^-6."""
    codes = torch.randint(low, high, weight[1].shape, generator=g).to(U8).to(DEV)
    return weight[0], codes, weight[2]


@pytest.mark.parametrize("t", [3, 40, 400])
@pytest.mark.parametrize("low, high, lost", [(-30.9, -28.0, 0.0), (-37.0, -35.0, 2.0 ** -39)])
def test_small_elements_of_x(t, low, high, lost):
    """x's largest elements meet zeros, so the others decide: exact down to 2^-31 of the largest, below it 2^-39 at most is lost."""
    n, inner, count, col = 256, 64, 5, 37
    g = torch.Generator().manual_seed(t)
    x = with_outlier(t, n, col, low, high, g)
    gate, up = (zero_column(matrices(count, inner, n, g, scale=1e-3 * 2.0 ** -high), col) for _ in range(2))
    down = matrices(count, n, inner, g)
    ids = torch.randint(count, (t, 2), generator=g).to(I32).to(DEV)
    w = (torch.rand(t, 2, generator=g) + 0.1).to(DEV)
    want, tol = experts(x.cpu(), ids.cpu(), w.cpu(), gate, up, down, 0)
    more = torch.zeros_like(tol)
    if lost:  # what g and u lose: its share of the largest times the sum of the weights' magnitudes
        for e in range(count):
            r, j = (ids.cpu() == e).nonzero(as_tuple=True)
            gm, um, dm = dequantized(gate, e), dequantized(up, e), dequantized(down, e)
            xe = x[r].cpu().double()
            a, u = activation(0, xe @ gm.T)[0], xe @ um.T
            dg, du = (lost * 1.5 * m.abs().sum(1) for m in (gm, um))
            dh = 1.13 * dg * (u.abs() + du) + a.abs() * du
            more.index_add_(0, r, w.cpu().double()[r, j][:, None] * (dh @ dm.abs().T))
    got = run(x, ids, w, gate, up, down, 0).cpu().double()
    assert ((got - want).abs() <= tol + 1.01 * more).all()
    # the tolerance is not what passes: the outputs are many times it
    assert (want.norm(dim=1) > 20 * (tol + more).norm(dim=1)).float().mean() > 0.9 or lost


@pytest.mark.parametrize("t", [3, 40, 400])
@pytest.mark.parametrize("kind", [0, 1])
def test_small_elements_of_h(t, kind):
    """h's largest elements, up to 2^32 times the others, meet zeros: 2^-11 of each element is lost, or 2^-38 of the largest."""
    n, inner, count, row = 256, 96, 5, 40
    g = torch.Generator().manual_seed(t)
    x, _ = rows(t, n, 0, g)
    gate, up = (far_codes(matrices(count, inner, n, g, scale=0.1), g) for _ in range(2))
    for m in (gate, up):
        m[1][:, row] = 126
    down = zero_column(matrices(count, n, inner, g), row)
    ids = torch.randint(count, (t, 2), generator=g).to(I32).to(DEV)
    w = (torch.rand(t, 2, generator=g) + 0.1).to(DEV)
    want, tol = experts(x.cpu(), ids.cpu(), w.cpu(), gate, up, down, kind)
    got = run(x, ids, w, gate, up, down, kind).cpu().double()
    assert ((got - want).abs() <= tol).all()
    assert (want.norm(dim=1) > 5 * tol.norm(dim=1)).float().mean() > 0.9


@pytest.mark.parametrize("t", [3, 40, 400])
@pytest.mark.parametrize("low, high", [(-30.9, -28.0), (-3.0, 0.0)])
def test_small_elements_of_dy_and_of_the_factors(t, low, high):
    """dy's largest elements meet zeros of D; the factors' largest ones, some 2^27 times the others, zeros of G."""
    n, inner, count, col, row = 256, 96, 5, 101, 40
    g = torch.Generator().manual_seed(t)
    dy = with_outlier(t, n, col, low, high, g)
    x, _ = rows(t, n, 0, g)
    gate, up = (far_codes(matrices(count, inner, n, g, scale=0.1), g) for _ in range(2))
    gate = zero_row(gate, row)   # act(0) = 0 and act'(0) = 1/2
    up[1][:, row] = 126
    down = zero_row(far_codes(matrices(count, n, inner, g, scale=0.1 * 2.0 ** -high), g), col)
    group = row // 16
    down[1][:, :, group] = 126
    packed = down[0].clone()
    packed[:, :, group * 8:group * 8 + 8] = 0
    packed[:, :, row // 2] = down[0][:, :, row // 2] & (0x0F if row % 2 == 0 else 0xF0)
    down = packed, down[1], down[2]
    ids = torch.randint(count, (t, 2), generator=g).to(I32).to(DEV)
    w = (torch.rand(t, 2, generator=g) + 0.1).to(DEV)
    dx, dw = backward(dy, x, ids, w, gate, up, down, 0)
    # In this row g = 0, act(g) = 0 and du = 0 exactly, and dg meets zeros: U's row takes no part in dx and dweights but by the
    # factors' common power of two, 2^-38 of the largest dg.
    rest = zero_row(up, row)
    want_dx, tol_dx, want_dw, tol_dw = experts_backward(dy.cpu(), x.cpu(), ids.cpu(), w.cpu(), gate, rest, down, 0)
    for e in range(count):
        r, j = (ids.cpu() == e).nonzero(as_tuple=True)
        dh, u = (dy[r].cpu().double() @ dequantized(down, e))[:, row], (x[r].cpu().double() @ dequantized(up, e).T)[:, row]
        largest = w.cpu().double()[r, j] * 0.5 * (dh * u).abs()
        tol_dx.index_add_(0, r, 2.0 ** -38 * largest[:, None] * (dequantized(gate, e).abs() + dequantized(rest, e).abs()).sum(0))
    assert ((dx.cpu().double() - want_dx).abs() <= tol_dx).all()
    assert ((dw.cpu().double() - want_dw).abs() <= tol_dw).all()
    assert (want_dx.norm(dim=1) > 5 * tol_dx.norm(dim=1)).float().mean() > 0.9


@pytest.mark.parametrize("t", [4, 50, 300])
@pytest.mark.parametrize("power", [-60, -31, 17, 50])
def test_far_scales_of_dy(t, power):
    """The gradients are linear in dy, and a power of two changes no bit of them."""
    x, ids, w, gate, up, down = layer(t, 272, 144, 5, 2, seed=3)
    dy, _ = rows(t, 272, 0, torch.Generator().manual_seed(4))
    dx, dw = backward(dy, x, ids, w, gate, up, down, 0)
    far_dx, far_dw = backward((dy.float() * 2.0 ** power).to(BF16), x, ids, w, gate, up, down, 0)
    assert torch.equal(far_dx.float(), dx.float() * 2.0 ** power) and torch.equal(far_dw, dw * 2.0 ** power)
