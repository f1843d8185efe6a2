"""The adapter operators as programs meet them: the example's training and serving, rows further than 2^32 elements
apart, and the projection's waits running out."""
import importlib.util
import pathlib

import pytest
import torch

import paper_2608_28113_gb300 as hs
from test_gpu_failure import both, starved  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
BF16, F64, U8, I32 = torch.bfloat16, torch.float64, torch.uint8, torch.int32
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


def test_the_example_trains_and_serves():
    path = pathlib.Path(__file__).resolve().parents[1] / "examples" / "adapter_step.py"
    spec = importlib.util.spec_from_file_location("adapter_step", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, served = example.run(m=256, n=512, tokens=512, steps=20)
    assert all(later < losses[0] for later in losses[5:]) and losses[-1] < 0.95 * losses[0]
    assert served.isfinite().all()
    assert not torch.equal(served[0], served[1])


def layer(m, n, count, rank, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    packed = torch.randint(256, (m, n // 2), generator=g, device=DEV, dtype=U8)
    codes = torch.randint(50, 80, (m, n // 16), generator=g, device=DEV, dtype=U8)
    sg = torch.full((1,), 1e-3, device=DEV)
    a = torch.randn(count, rank, n, generator=g, device=DEV).to(BF16)
    b = torch.randn(count, m, rank, generator=g, device=DEV).to(BF16)
    return packed, codes, sg, a, b, torch.ones(count, device=DEV)


@pytest.mark.parametrize("t", [16, 20])
def test_rows_far_apart(t):
    """Rows 2^28 + 64 elements apart: the last ones begin past 2^32 (bytes and, from 17 rows on, elements)."""
    m, n, ld = 96, 128, (1 << 28) + 64
    if torch.cuda.mem_get_info()[0] < 2.5 * t * ld:
        pytest.skip("not enough memory")
    packed, codes, sg, a, b, alpha = layer(m, n, 3, 16)
    g = torch.Generator(device=DEV).manual_seed(1)
    ids = torch.randint(-1, 3, (t,), generator=g, device=DEV).to(I32)
    far = torch.empty(t * ld, dtype=BF16, device=DEV).view(t, ld)
    x, y, dy, dx = far[:, :n], far[:, n:n + m], far[:, 256:256 + m], far[:, 384:384 + n]
    x.copy_(torch.randn(t, n, generator=g, device=DEV))
    dy.copy_(torch.randn(t, m, generator=g, device=DEV))
    q, s = far.view(torch.uint8)[:, 2048:2048 + n], far.view(torch.uint8)[:, 4096:4096 + n // 32]
    hs.hscale_checkpoint_save(x, 0, q, s)
    da, db = torch.empty_like(a), torch.empty_like(b)
    hs.hscale_project(x, packed, codes, sg, a, b, alpha, ids, y)
    hs.hscale_project_backward(dy, q, s, 0, packed, codes, sg, a, b, alpha, ids, dx, da, db)
    xc, dyc, qc, sc = x.contiguous(), dy.contiguous(), q.contiguous(), s.contiguous()
    near_q, near_s = torch.empty_like(qc), torch.empty_like(sc)
    hs.hscale_checkpoint_save(xc, 0, near_q, near_s)
    assert torch.equal(qc, near_q) and torch.equal(sc, near_s)
    near_y, near_dx, near_da, near_db = (torch.empty(t, m, dtype=BF16, device=DEV), torch.empty_like(xc), torch.empty_like(a),
                                         torch.empty_like(b))
    hs.hscale_project(xc, packed, codes, sg, a, b, alpha, ids, near_y)
    hs.hscale_project_backward(dyc, qc, sc, 0, packed, codes, sg, a, b, alpha, ids, near_dx, near_da, near_db)
    assert torch.equal(y.contiguous(), near_y) and torch.equal(dx.contiguous(), near_dx)
    assert torch.equal(da, near_da) and torch.equal(db, near_db)


@pytest.mark.parametrize("t, m, n", [(20000, 384, 640), (300, 128, 4096), (64, 2048, 2048)])  # persistent, and clusters
def test_projection_of_a_starved_block(starved, monkeypatch, t, m, n):  # noqa: F811
    """The tiles of a block whose epilogue gives up are NaN, all of them; the others are what they were."""
    packed, codes, sg, a, b, alpha = layer(m, n, 2, 16, seed=2)
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(t, n, generator=g, device=DEV).to(BF16)
    ids = torch.randint(-1, 2, (t,), generator=g, device=DEV).to(I32)

    def call():
        y = torch.zeros(t, m, dtype=BF16, device=DEV)
        hs.hscale_project(x, packed, codes, sg, a, b, alpha, ids, y)
        return y

    got, want = both(starved, monkeypatch, call)
    lost = got.isnan()
    assert lost.any() and not want.isnan().any()
    assert torch.equal(got[~lost], want[~lost])
    # whole tiles: 128 outputs (or what is left) of the tokens concerned
    for c in range(0, m, 128):
        part = lost[:, c:c + 128]
        assert torch.equal(part.all(1), part.any(1))
