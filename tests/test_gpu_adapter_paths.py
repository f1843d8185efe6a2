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


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("rank", [8, 32, 64])
@pytest.mark.parametrize("lead, pad, scale_lead, scale_pad", [(8, 8, 0, 0), (1, 3, 0, 0), (0, 0, 1, 2), (5, 4, 3, 1)])
def test_checkpoint_rows_at_any_address(fmt, rank, lead, pad, scale_lead, scale_pad):
    """The gradients read codes and scales at any address, and get the same bits as from aligned ones."""
    t, m, n, count = 150, 96, 400, 3
    packed, codes, sg, a, b, alpha = layer(m, n, count, rank, seed=4)
    g = torch.Generator(device=DEV).manual_seed(5)
    ids = torch.randint(-1, count, (t,), generator=g, device=DEV).to(I32)
    dy = torch.randn(t, m, generator=g, device=DEV).to(BF16)
    q, s = torch.empty(t, n, dtype=U8, device=DEV), torch.empty(t, (n + 31) // 32, dtype=U8, device=DEV)
    hs.hscale_checkpoint_save(torch.randn(t, n, generator=g, device=DEV).to(BF16), fmt, q, s)

    def gradients(q, s):
        dx = torch.empty(t, n, dtype=BF16, device=DEV)
        da, db = torch.empty_like(a), torch.empty_like(b)
        hs.hscale_project_backward(dy, q, s, fmt, packed, codes, sg, a, b, alpha, ids, dx, da, db)
        return dx, da, db

    def moved(v, lead, pad):
        rows, cols = v.shape
        wide = torch.randint(256, (lead + rows * (cols + pad),), generator=g, device=DEV, dtype=U8)
        view = wide[lead:].view(rows, cols + pad)[:, :cols]
        view.copy_(v)
        return view

    for got, want in zip(gradients(moved(q, lead, pad), moved(s, scale_lead, scale_pad)), gradients(q, s)):
        assert torch.equal(got, want) and want.float().abs().max() > 0


@pytest.mark.parametrize("t, order", [(7, "any"), (64, "each its own"), (257, "any"), (700, "runs"), (520, "rare")])
def test_gradients_of_many_adapters(t, order):
    """More adapters than a tile lists or an SM has CTAs, most of them with few tokens or none, against the formulas in 64
    bits.  Tolerance: dA and dB are rounded once to bf16, at most 2^-8 of a value.  Before that, in units of the terms'
    summed magnitudes: z and dz are fp32 sums of at most 272 terms (272 2^-24) that enter as pairs (2^-17), and the
    tokens, at most 520 of an adapter, are summed in fp32 (520 2^-23): together less than 2^-13."""
    m, n, count, rank = 136, 272, 300, 8
    packed, codes, sg, a, b, alpha = layer(m, n, count, rank, seed=6)
    g = torch.Generator(device=DEV).manual_seed(7)
    ids = {"any": torch.randint(-1, count, (t,), generator=g, device=DEV),
           "each its own": torch.randperm(count, generator=g, device=DEV)[:t],
           "runs": torch.arange(t, device=DEV) // 3 % count,
           "rare": torch.where(torch.arange(t, device=DEV) % 97 == 0, torch.arange(t, device=DEV) % count, count - 1)}[order].to(I32)
    dy = torch.randn(t, m, generator=g, device=DEV).to(BF16)
    q, s = torch.empty(t, n, dtype=U8, device=DEV), torch.empty(t, (n + 31) // 32, dtype=U8, device=DEV)
    x = torch.empty(t, n, dtype=BF16, device=DEV)
    hs.hscale_checkpoint_save(torch.randn(t, n, generator=g, device=DEV).to(BF16), 0, q, s)
    hs.hscale_checkpoint_load(q, s, 0, x)
    da, db = torch.empty_like(a), torch.empty_like(b)
    hs.hscale_project_backward(dy, q, s, 0, packed, codes, sg, a, b, alpha, ids, None, da, db)
    on = (ids >= 0).nonzero()[:, 0]
    who, xd, dyd = ids[on].long(), x[on].to(F64), dy[on].to(F64)
    ad, bd = a.to(F64)[who], b.to(F64)[who]
    z, dz = torch.einsum("trn,tn->tr", ad, xd), torch.einsum("tmr,tm->tr", bd, dyd)
    for got, left, right, inner in ((da, dz, xd, torch.einsum("tmr,tm->tr", bd.abs(), dyd.abs())),
                                    (db, dyd, z, torch.einsum("trn,tn->tr", ad.abs(), xd.abs()))):
        want = torch.zeros(got.shape, dtype=F64, device=DEV).index_add_(0, who, left[:, :, None] * right[:, None, :])
        size_l, size_r = (inner, right.abs()) if got is da else (left.abs(), inner)
        size = torch.zeros(got.shape, dtype=F64, device=DEV).index_add_(0, who, size_l[:, :, None] * size_r[:, None, :])
        assert bool(((got.to(F64) - want).abs() <= want.abs() / 2**8 + size / 2**13).all())
        idle = torch.ones(count, dtype=torch.bool, device=DEV)
        idle[who] = False
        assert not got[idle].any()
