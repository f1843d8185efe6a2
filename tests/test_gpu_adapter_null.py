"""The backward pass where adapter_of is not given: every token is on adapter 0, and the other adapters have none."""
import pytest
import torch

import paper_2608_28113_gb300 as hs
from test_gpu_adapters import BF16, DEV, F64, I32, Layer, check, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("t, m, n, count, rank", [
    (1, 24, 32, 2, 8), (16, 130, 400, 3, 16), (40, 72, 96, 5, 24), (300, 264, 528, 3, 32), (700, 129, 176, 2, 64),
    (300, 200, 272, 40, 128)])
def test_adapters_without_tokens_get_zeros(t, m, n, count, rank, fmt):
    """Adapter 0's gradients against the formulas in 64 bits (the tolerances of test_gpu_adapters), the others' zero."""
    L = Layer(t, m, n, count, rank, None, fmt=fmt)
    check(L.project(), L.forward64(), L.forward64(absolute=True), n + rank)
    dx, da, db, held = L.backward()
    wx, wa, wb = L.backward64(held)
    sx, sa, sb = L.backward64(held, absolute=True)
    assert not wa[1:].any() and not wb[1:].any()
    check(dx, wx, sx, 2 * m + rank)
    check(da, wa, sa, t + m, 2.0 ** -16)
    check(db, wb, sb, t + n, 2.0 ** -16)
    assert not da[1:].any() and not db[1:].any()


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("t, m, n", [(9000, 5120, 5120), (8200, 9984, 256)])
def test_windows_of_tokens_follow_one_another(t, m, n, fmt):
    """Tokens are taken in windows of 4096, here by clusters of three, whose CTAs end a window on different chunks.  The
    tokens' magnitudes differ by powers of two, so that one token's scales on another's elements show.  dA and dB
    against the formulas in 64 bits (the tolerances of test_gpu_adapters), the bits of a call that names adapter 0 for each
    token, and the same bits again."""
    L = Layer(t, m, n, 1, 16, None, fmt=fmt)
    L.x.mul_(torch.exp2(torch.randint(-12, 13, (t, 1), generator=gen("magnitudes", t, fmt), device=DEV)).to(BF16))
    dx, da, db, held = L.backward()
    x, dy, a, b, alpha = held.to(F64), L.dy.to(F64), L.a[0].to(F64), L.b[0].to(F64), L.alpha[0].to(F64)
    dz, z = alpha * dy @ b, alpha * x @ a.T
    check(da[0], dz.T @ x, (alpha * dy.abs() @ b.abs()).T @ x.abs(), t + m, 2.0 ** -16)
    check(db[0], dy.T @ z, dy.abs().T @ (alpha * x.abs() @ a.abs().T), t + n, 2.0 ** -16)
    for _ in range(4):
        again = L.backward()
        assert torch.equal(again[1], da) and torch.equal(again[2], db)
    L.ids = torch.zeros(t, dtype=I32, device=DEV)
    named = L.backward()
    for got, want in zip(named[:3], (dx, da, db)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("t, m, n, rank, fmt", [(2000, 2048, 2048, 64, 0), (1000, 1024, 4096, 16, 1), (200, 4096, 4096, 8, 0)])
def test_adapters_without_tokens_change_nothing(t, m, n, rank, fmt):
    """However many adapters there are beside adapter 0, its gradients are dealt out, and summed, alike: the same bits."""
    L = Layer(t, m, n, 40, rank, None, fmt=fmt)
    y, (dx, da, db, _) = L.project(), L.backward()
    L.count, L.a, L.b, L.alpha = 1, L.a[:1].contiguous(), L.b[:1].contiguous(), L.alpha[:1].contiguous()
    alone = L.backward()
    assert torch.equal(L.project(), y) and torch.equal(alone[0], dx)
    assert torch.equal(alone[1][0], da[0]) and torch.equal(alone[2][0], db[0])
