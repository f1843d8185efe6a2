"""The sums behind dweights are as exact from long rows as from short ones."""
import pytest
import torch

import paper_2608_28113_gb300 as hs
from expert_reference import experts_backward
from test_gpu_experts import backward, clean, layer, moved, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


@pytest.mark.parametrize("n", [4096, 8192, 16384])
@pytest.mark.parametrize("packed_by, codes_by", [(0, 0), (8, 4), (16, 1)])
def test_dweights_of_long_rows_are_as_exact_as_of_short_ones(n, packed_by, codes_by):
    """Parts of 1024 columns (g, u) and at most 1408 (dh) are summed up from zero: each loses the share of its sum that a row as
    long does, so dweights at most 1408 / 1024 = 1.375 times what a row of 1024 columns loses; the sums of up to 16 parts, rounded at
    random, add less than 2 2^-24 to some 20 of them.  Whole sums lose 5 times as much at 4096 columns, 25 at 16384."""
    t, inner, count, k = 350, 80, 2, 2

    def error(cols):
        x, ids, w, gate, up, down = layer(t, cols, inner, count, k, seed=cols)
        gate, up, down = (moved(m, packed_by, codes_by) for m in (gate, up, down))
        dy, _ = rows(t, cols, 16, torch.Generator().manual_seed(8), 0.1)
        _, dw = backward(dy, x, ids, w, gate, up, down, 0)
        _, _, want, _ = experts_backward(dy.cpu(), x.cpu(), ids.cpu(), clean(w), gate, up, down, 0)
        return ((dw.cpu().double() - want).norm() / want.norm()).item()

    assert error(n) <= 1.5 * error(1024)
