"""What a token's gradients share with the rest of its batch: dweights has the same bits in any batch, dx in any batch
of as many tokens (how G's and U's parts of it are added goes by the sizes)."""
import pytest
import torch

import paper_2608_28113_gb300 as hs
from test_gpu_experts import backward, clean, layer, rows
from expert_reference import experts_backward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


# few and many columns of dx (so the last round of tiles is filled more or less), one segment of K and several, rows of
# whole 32 columns and not
SIZES = [(448, 208, 5), (4096, 208, 5), (4112, 272, 5), (1600, 1616, 3)]


@pytest.mark.parametrize("n, inner, count", SIZES)
def test_dweights_do_not_depend_on_the_batch(n, inner, count):
    args = layer(900, n, inner, count, 2, seed=31)
    x, ids, w, gate, up, down = args
    dy, _ = rows(900, n, 0, torch.Generator().manual_seed(2))
    dx, dw = backward(dy, *args, 0)
    for start, tokens in ((0, 1), (17, 12), (100, 90), (300, 400)):
        part = slice(start, start + tokens)
        some = dy[part], x[part], ids[part].contiguous(), w[part].contiguous()
        got_dx, got_dw = backward(*some, gate, up, down, 0)
        assert torch.equal(got_dw, dw[part])
        # dx: each within the bound, so at most twice the bound apart
        _, tol, _, _ = experts_backward(some[0].cpu(), some[1].cpu(), some[2].cpu(), clean(some[3]), gate, up, down, 0)
        assert ((got_dx.cpu().double() - dx[part].cpu().double()).abs() <= 2 * tol).all()


@pytest.mark.parametrize("n, inner, count", SIZES)
@pytest.mark.parametrize("t", [20, 900])
def test_gradients_do_not_depend_on_the_other_tokens(n, inner, count, t):
    args = layer(t, n, inner, count, 2, seed=31)
    x, ids, w, gate, up, down = args
    dy, _ = rows(t, n, 0, torch.Generator().manual_seed(2))
    dx, dw = backward(dy, *args, 0)
    # the others on other experts, with other values
    kept = torch.arange(t, device=x.device) % 7 == 3
    other = [torch.where(kept[:, None], v, v.roll(1, 1)).contiguous() for v in (dy, x)]
    moved = torch.where(kept[:, None], ids, ids * 0 + count - 1)
    got_dx, got_dw = backward(*other, moved, w, gate, up, down, 0)
    assert torch.equal(got_dx[kept], dx[kept]) and torch.equal(got_dw[kept], dw[kept])
    alone_dx, _ = backward(*other, moved, w, gate, up, down, 0, want_dw=False)
    assert torch.equal(alone_dx[kept], dx[kept])
