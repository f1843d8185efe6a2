"""The gradients' norm over so many elements that a thread adds up thousands of pieces."""
import math

import pytest
import torch

import paper_2608_28113_gb300 as hs

pytestmark = pytest.mark.gpu


# Equal elements: each addition to a long fp32 sum is rounded the same way, so the errors add up.  A tensor is read as many
# times as it is listed: (value, times it is listed); 2^28 elements are some 108 pieces of 16 a thread.
@pytest.mark.parametrize("value, times", [(0.9, 47), (1.1, 187), (1.1 * 2.0 ** 80, 12), (1.3 * 2.0 ** -60, 12), (0.9 * 2.0 ** 80, 47)])
def test_long_sums(value, times):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()
    if torch.cuda.mem_get_info()[0] < 3 << 30:
        pytest.skip("not enough memory")
    part = torch.full((1 << 28,), value, device="cuda")
    norm = torch.empty(1, device="cuda")
    hs.hscale_grad_norm([part] * times, norm)
    want = part[0].double().item() * math.sqrt(times * 2.0 ** 28)
    # a piece's 16 squares and at most 64 pieces are added up in fp32, the rest in fp64: 80 roundings of the sum of the squares,
    # half of that of its root, and the root's own
    assert abs(norm.item() - want) <= want * 41 * 2.0 ** -24
