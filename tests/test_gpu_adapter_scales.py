"""The projection with adapters under global scales far from the adapters' magnitudes.  On the tensor cores the adapters'
terms are summed with the weight's, in units of the global scale."""
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


@pytest.mark.parametrize("sg", [0.0, 2.0 ** -140, 1e-37, -1e-30, 1e-12, -0.5, 1e12, 1e30])
@pytest.mark.parametrize("t, m, n, count, rank, ids", [
    (5, 130, 272, 2, 16, "mixed"), (48, 200, 2048, 2, 16, "runs"), (300, 264, 528, 3, 32, "runs"), (700, 264, 272, 3, 8, "mixed"),
    (6000, 640, 512, 2, 64, "runs")])
def test_any_global_scale(t, m, n, count, rank, ids, sg):
    """Against 64 bits, with the tolerances of test_gpu_adapters and 2^-17 of the terms' magnitudes for z and dz as pairs of
    bf16 numbers."""
    L = Layer(t, m, n, count, rank, ids)
    L.sg.fill_(sg)
    check(L.project(), L.forward64(), L.forward64(absolute=True), n + rank, 2.0 ** -17)
    dx, _, _, held = L.backward(("dx",))
    check(dx, L.backward64(held)[0], L.backward64(held, absolute=True)[0], 2 * m + rank, 2.0 ** -17)
