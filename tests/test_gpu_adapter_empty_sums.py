"""The gradients of a projection without outputs (m == 0) whose matrices are really empty: what exists of them is zero."""
import pytest
import torch

import paper_2608_28113_gb300 as hs
from test_gpu_adapters import BF16, DEV, F32, I32, U8, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", [1, 4, 300])
@pytest.mark.parametrize("ids", [True, False])
def test_no_outputs(t, ids):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    n, count, rank = 64, 2, 16

    def empty(*shape, dtype=BF16):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    dy, packed, codes, b = empty(t, 0), empty(0, n // 2, dtype=U8), empty(0, n // 16, dtype=U8), empty(count, 0, rank)
    assert dy.data_ptr() == 0
    a, dx = torch.ones(count, rank, n, dtype=BF16, device=DEV), rows(t, n, n + 8)
    da, db = torch.full_like(a, float("nan")), torch.empty_like(b)
    x, scales = torch.ones(t, n, dtype=U8, device=DEV), torch.full((t, 2), 127, dtype=U8, device=DEV)
    who = torch.zeros(t, dtype=I32, device=DEV) if ids else None
    one = torch.ones(1, dtype=F32, device=DEV)
    hs.hscale_project_backward(dy, x, scales, 0, packed, codes, one, a, b, one.expand(count).contiguous(), who, dx, da, db)
    assert (dx == 0).all() and (da == 0).all()
    assert t == 1 or dx.as_strided((t, 8), (n + 8, 1), n)[:-1].isnan().all()
