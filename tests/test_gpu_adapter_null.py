"""The backward pass where adapter_of is not given: every token is on adapter 0, and the other adapters have none."""
import pytest
import torch

import paper_2608_28113_gb300 as hs
from test_gpu_adapters import Layer, check

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
