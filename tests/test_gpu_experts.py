"""A layer of packed experts and its gradients against plain 64-bit operations."""
import math

import pytest
import torch

import paper_2608_28113_gb300 as hs
from expert_reference import experts, experts_backward

pytestmark = pytest.mark.gpu
BF16, F32, F64, U8, I32 = torch.bfloat16, torch.float32, torch.float64, torch.uint8, torch.int32
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


def matrices(count, rows, cols, g, scale=1e-3):
    packed = torch.randint(256, (count, rows, cols // 2), generator=g, dtype=torch.int64).to(U8)
    codes = torch.randint(40, 80, (count, rows, cols // 16), generator=g, dtype=torch.int64).to(U8)
    codes[torch.rand(codes.shape, generator=g) < 0.02] = 0      # read as 1
    codes[torch.rand(codes.shape, generator=g) < 0.02] = 255    # read as 126 (the sign bit is ignored)
    codes[codes == 255] = 70 + 128
    sg = scale * (0.5 + torch.rand(count, generator=g))
    return packed.to(DEV), codes.to(DEV), sg.to(DEV)


def rows(t, n, pad, g, scale=1.0):
    full = torch.full((t, (n + pad + 7) // 8 * 8), 3.0, dtype=BF16, device=DEV)
    full[:, :n] = (torch.randn(t, n, generator=g) * scale).to(BF16)
    return full[:, :n], full


def layer(t, n, inner, count, k, seed=0, pad=8, none=0.1, skew=0):
    g = torch.Generator().manual_seed(seed)
    x, _ = rows(t, n, pad, g)
    gate, up, down = matrices(count, inner, n, g), matrices(count, inner, n, g), matrices(count, n, inner, g)
    ids = torch.randint(count, (t, k), generator=g)
    if skew:
        ids = torch.where(torch.rand(t, k, generator=g) < 0.9, torch.full_like(ids, skew % count), ids)
    ids = torch.where(torch.rand(t, k, generator=g) < none, torch.randint(-3, 0, (t, k), generator=g), ids)
    ids = torch.where(torch.rand(t, k, generator=g) < none / 3, count + 5, ids).to(I32)
    w = torch.rand(t, k, generator=g) + 0.1
    w[(ids < 0) | (ids >= count)] = math.nan  # a weight that no expert goes by
    return x, ids.to(DEV), w.to(DEV), gate, up, down


# tokens, n, inner, experts, k
SIZES = [(1, 16, 16, 1, 1), (1, 64, 32, 4, 2), (1, 512, 256, 16, 8), (3, 80, 48, 5, 3), (37, 272, 144, 12, 3), (64, 128, 128, 64, 8),
         (130, 512, 256, 8, 2), (300, 256, 400, 3, 2), (600, 64, 80, 2, 1), (45, 1040, 528, 40, 4), (9, 2048, 64, 1024, 32),
         (70, 144, 1040, 7, 5), (1100, 320, 192, 2, 2), (640, 256, 512, 1, 1), (1300, 64, 48, 40, 8)]


def clean(w):
    return torch.where(torch.isnan(w), 0.0, w).cpu()


def run(x, ids, w, gate, up, down, kind, **kwargs):
    t, n = x.shape
    full = torch.full((t, n + 16), 5.0, dtype=BF16, device=DEV)
    hs.hscale_experts(x, ids, w, gate, up, down, kind, full[:, :n], **kwargs)
    torch.cuda.current_stream().synchronize()
    assert (full[:, n:] == 5.0).all()
    return full[:, :n]


@pytest.mark.parametrize("t, n, inner, count, k", SIZES)
@pytest.mark.parametrize("kind", [0, 1])
def test_experts(t, n, inner, count, k, kind):
    args = layer(t, n, inner, count, k, seed=t + n)
    y = run(*args, kind)
    x, ids, w, gate, up, down = args
    want, tol = experts(x.cpu(), ids.cpu(), clean(w), gate, up, down, kind)
    got = y.cpu().double()
    assert ((got - want).abs() <= tol).all()
    norm = want.norm()
    if norm > 0:  # y off by at most 2^-8, h by 2^-11, which sums of many leave the same
        assert (got - want).norm() <= norm * 1.5 * 2.0 ** -8
    assert torch.equal(run(*args, kind), y)
    assert hs.hscale_device_error_flags() == 0


def backward(dy, x, ids, w, gate, up, down, kind, want_dx=True, want_dw=True, **kwargs):
    t, n = x.shape
    full = torch.full((t, n + 8), 5.0, dtype=BF16, device=DEV)
    dw = torch.full(w.shape, math.nan, device=DEV)
    hs.hscale_experts_backward(dy, x, ids, w, gate, up, down, kind, full[:, :n] if want_dx else None, dw if want_dw else None, **kwargs)
    torch.cuda.current_stream().synchronize()
    assert (full[:, n:] == 5.0).all()
    return full[:, :n], dw


@pytest.mark.parametrize("t, n, inner, count, k", SIZES)
@pytest.mark.parametrize("kind", [0, 1])
def test_experts_backward(t, n, inner, count, k, kind):
    args = layer(t, n, inner, count, k, seed=t + n)
    x, ids, w, gate, up, down = args
    dy, _ = rows(t, n, 16, torch.Generator().manual_seed(8), 0.1)
    dx, dw = backward(dy, *args, kind)
    want_dx, tol_dx, want_dw, tol_dw = experts_backward(dy.cpu(), x.cpu(), ids.cpu(), clean(w), gate, up, down, kind)
    assert ((dx.cpu().double() - want_dx).abs() <= tol_dx).all()
    assert ((dw.cpu().double() - want_dw).abs() <= tol_dw).all()
    if want_dx.norm() > 0:
        assert (dx.cpu().double() - want_dx).norm() <= want_dx.norm() * 1.5 * 2.0 ** -8
    again = backward(dy, *args, kind)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    alone_dx, _ = backward(dy, *args, kind, want_dw=False)
    _, alone_dw = backward(dy, *args, kind, want_dx=False)
    assert torch.equal(alone_dx, dx) and torch.equal(alone_dw, dw)
    assert hs.hscale_device_error_flags() == 0


@pytest.mark.parametrize("t, n, inner, count, k", [(90, 4176, 272, 3, 2), (20, 5632, 144, 6, 2), (700, 8192, 80, 2, 2), (40, 1424, 528, 2, 3)])
@pytest.mark.parametrize("packed_by, codes_by", [(0, 0), (8, 4), (16, 1)])
def test_backward_of_long_rows(t, n, inner, count, k, packed_by, codes_by):
    """g, u and dh are summed in parts: dweights is as exact from long rows as from short ones."""
    x, ids, w, gate, up, down = layer(t, n, inner, count, k, seed=n)
    gate, up, down = (moved(m, packed_by, codes_by) for m in (gate, up, down))
    dy, _ = rows(t, n, 16, torch.Generator().manual_seed(8), 0.1)
    dx, dw = backward(dy, x, ids, w, gate, up, down, 0)
    want_dx, tol_dx, want_dw, tol_dw = experts_backward(dy.cpu(), x.cpu(), ids.cpu(), clean(w), gate, up, down, 0)
    assert ((dx.cpu().double() - want_dx).abs() <= tol_dx).all()
    assert ((dw.cpu().double() - want_dw).abs() <= tol_dw).all()
    # An accumulator of fp32 that is cut off toward zero at each step of 16: half a unit of 2^-23 on average, 0.72 of it relative
    # to the sum (a mantissa's mean reciprocal), and the partial sums of random products grow as a square root: of m steps
    # 0.36 2^-23 sum_j sqrt(j / m) = 0.48 m 2^-24.  Parts of at most 1408 columns of g and u and of 2048 of dh: m = 88, 88 and
    # 128, together 146 2^-24, however long the rows are (shorter parts lose less).  The roundings of the parts' sums, of the activation, of the
    # products and of their sum over inner, each random: less than 14 2^-24.
    assert (dw.cpu().double() - want_dw).norm() <= want_dw.norm() * 160 * 2.0 ** -24
    again = backward(dy, x, ids, w, gate, up, down, 0)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    assert hs.hscale_device_error_flags() == 0


@pytest.mark.parametrize("t", [1, 20, 200])
def test_tokens_do_not_meet(t):
    """Inf and NaN in some rows, some weights and the factors of an expert that few tokens are on stay with them."""
    x, ids, w, gate, up, down = layer(t, 128, 96, 6, 2, seed=5, none=0.2)
    dy, _ = rows(t, 128, 0, torch.Generator().manual_seed(1))
    gate[2][5] = math.inf
    down[2][4] = math.nan
    w = torch.where(torch.isnan(w), 0.5, w)
    w[::7, 0] = math.inf
    bad_row = torch.zeros(t, dtype=torch.bool, device=DEV)
    bad_row[1::5] = True
    x = x.clone()
    x[bad_row] = math.nan
    dirty = bad_row | ((ids == 5) | (ids == 4)).any(1)
    dirty[::7] = True
    y = run(x, ids, w, gate, up, down, 0)
    dx, dw = backward(dy, x, ids, w, gate, up, down, 0)
    clean_x = torch.where(bad_row[:, None], 0.0, x.float()).to(BF16)
    keep = ~dirty
    if not keep.any():
        return
    want, tol = experts(clean_x[keep].cpu(), ids[keep].cpu(), w[keep].cpu(), gate, up, down, 0)
    want_dx, tol_dx, want_dw, tol_dw = experts_backward(dy[keep].cpu(), clean_x[keep].cpu(), ids[keep].cpu(), w[keep].cpu(), gate, up,
                                                        down, 0)
    finite = ~want.isnan()
    assert finite.all()
    assert ((y[keep].cpu().double() - want).abs() <= tol).all()
    assert ((dx[keep].cpu().double() - want_dx).abs() <= tol_dx).all()
    assert ((dw[keep].cpu().double() - want_dw).abs() <= tol_dw).all()


@pytest.mark.parametrize("t", [2, 60, 300])
def test_no_expert_at_all(t):
    x, ids, w, gate, up, down = layer(t, 64, 48, 4, 3)
    ids.fill_(-1)
    y = run(x, ids, w, gate, up, down, 0)
    dx, dw = backward(x, x, ids, w, gate, up, down, 0)
    assert (y == 0).all() and (dx == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("t, count, k", [(5, 6, 4), (40, 6, 4), (150, 6, 4)])
def test_one_expert_has_nearly_all(t, count, k):
    """Uneven experts, the same one several times in a token among them."""
    args = layer(t, 192, 112, count, k, seed=11, skew=3)
    x, ids, w, gate, up, down = args
    want, tol = experts(x.cpu(), ids.cpu(), clean(w), gate, up, down, 1)
    assert ((run(*args, 1).cpu().double() - want).abs() <= tol).all()
    dy, _ = rows(t, 192, 0, torch.Generator().manual_seed(2))
    dx, dw = backward(dy, *args, 1)
    want_dx, tol_dx, want_dw, tol_dw = experts_backward(dy.cpu(), x.cpu(), ids.cpu(), clean(w), gate, up, down, 1)
    assert ((dx.cpu().double() - want_dx).abs() <= tol_dx).all()
    assert ((dw.cpu().double() - want_dw).abs() <= tol_dw).all()


@pytest.mark.parametrize("t", [4, 50, 260])
@pytest.mark.parametrize("scale", [2.0 ** -40, 2.0 ** 30])
def test_far_scales_of_x(t, scale):
    """x far from 1: its bf16 range is wider than 16-bit floats'.  gate's scale undoes it."""
    x, ids, w, gate, up, down = layer(t, 256, 64, 5, 2, seed=3)
    want, tol = experts(x.cpu(), ids.cpu(), clean(w), gate, up, down, 0)
    moved = (x.float() * scale).to(BF16)
    gate, up = (gate[0], gate[1], gate[2] / scale), (up[0], up[1], up[2] / scale)
    y = run(moved, ids, w, gate, up, down, 0)
    assert ((y.cpu().double() - want).abs() <= tol).all()


@pytest.mark.parametrize("t", [4, 100])
def test_streams_and_graphs(t):
    args = layer(t, 256, 128, 8, 2, seed=6)
    dy, _ = rows(t, 256, 0, torch.Generator().manual_seed(2))
    want, (want_dx, want_dw) = run(*args, 0), backward(dy, *args, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = torch.empty_like(want)
    hs.hscale_experts(*args, 0, y, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    with torch.cuda.stream(side):
        assert torch.equal(run(*args, 0), want)
    torch.cuda.synchronize()
    x, ids, w, gate, up, down = args
    n, inner, count, k = 256, 128, 8, 2
    y1, dx1, dw1 = torch.empty_like(want), torch.empty_like(want_dx), torch.empty_like(want_dw)
    ws = torch.empty(hs.hscale_experts_workspace_bytes(t, k, n, inner, count), dtype=U8, device=DEV)
    wsb = torch.empty(hs.hscale_experts_backward_workspace_bytes(t, k, n, inner, count), dtype=U8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hs.hscale_experts(*args, 0, y1, ws)
        hs.hscale_experts_backward(dy, *args, 0, dx1, dw1, wsb)
    # other tokens and experts than at the capture
    x.copy_(torch.roll(x, 1, 1))
    ids.copy_(torch.roll(ids, 1, 0))
    w.copy_(torch.where(torch.isnan(torch.roll(w, 1, 0)), 0.25, torch.roll(w, 1, 0)))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y1, run(*args, 0))
    dx, dw = backward(dy, *args, 0)
    assert torch.equal(dx1, dx) and torch.equal(dw1, dw)


def moved(weight, packed_by, codes_by):
    """The same weight at other addresses: bytes behind a multiple of 256."""
    out = []
    for t, by in zip(weight[:2], (packed_by, codes_by)):
        room = torch.empty(t.numel() + by, dtype=U8, device=DEV)
        room[by:] = t.reshape(-1)
        out.append(room[by:].view(t.shape))
    return out[0], out[1], weight[2]


@pytest.mark.parametrize("t, n, inner", [(5, 256, 512), (150, 512, 256), (5, 96, 160), (150, 320, 96), (150, 272, 176), (1100, 256, 272)])
@pytest.mark.parametrize("packed_by, codes_by", [(8, 0), (16, 4), (8, 4), (0, 1), (24, 6)])
def test_weights_at_any_address(t, n, inner, packed_by, codes_by):
    """Each way that the packed weights come to be unpacked gives the same bits."""
    x, ids, w, gate, up, down = layer(t, n, inner, 4, 2, seed=21)
    dy, _ = rows(t, n, 0, torch.Generator().manual_seed(2))
    want, (want_dx, want_dw) = run(x, ids, w, gate, up, down, 0), backward(dy, x, ids, w, gate, up, down, 0)
    other = [moved(m, packed_by, codes_by) for m in (gate, up, down)]
    assert torch.equal(run(x, ids, w, *other, 0), want)
    dx, dw = backward(dy, x, ids, w, *other, 0)
    assert torch.equal(dx, want_dx) and torch.equal(dw, want_dw)


@pytest.mark.parametrize("t, n, inner, count, k", [(3, 8208, 32, 3, 2), (70, 16400, 48, 2, 2), (40, 64, 9232, 3, 2), (300, 80, 8200 // 16 * 16, 2, 1)])
def test_rows_longer_than_registers_hold(t, n, inner, count, k):
    """x and dy past the 8192 columns that a CTA keeps, h and the factors past them."""
    args = layer(t, n, inner, count, k, seed=t)
    x, ids, w, gate, up, down = args
    want, tol = experts(x.cpu(), ids.cpu(), clean(w), gate, up, down, 1)
    assert ((run(*args, 1).cpu().double() - want).abs() <= tol).all()
    dy, _ = rows(t, n, 16, torch.Generator().manual_seed(8), 0.1)
    dx, dw = backward(dy, *args, 1)
    want_dx, tol_dx, want_dw, tol_dw = experts_backward(dy.cpu(), x.cpu(), ids.cpu(), clean(w), gate, up, down, 1)
    assert ((dx.cpu().double() - want_dx).abs() <= tol_dx).all()
    assert ((dw.cpu().double() - want_dw).abs() <= tol_dw).all()
    assert hs.hscale_device_error_flags() == 0


@pytest.mark.parametrize("t", [3, 40, 300])
def test_in_place(t):
    """y over x, and dx over dy and over x."""
    x, ids, w, gate, up, down = layer(t, 272, 144, 4, 2, seed=31)
    dy, _ = rows(t, 272, 0, torch.Generator().manual_seed(2))
    want, (want_dx, want_dw) = run(x, ids, w, gate, up, down, 0), backward(dy, x, ids, w, gate, up, down, 0)
    y = x.clone()
    hs.hscale_experts(y, ids, w, gate, up, down, 0, y)
    assert torch.equal(y, want)
    for onto_x in (False, True):
        dw, a, b = torch.zeros_like(w), dy.clone(), x.clone()
        dx = b if onto_x else a
        hs.hscale_experts_backward(a, b, ids, w, gate, up, down, 0, dx, dw)
        assert torch.equal(dx, want_dx) and torch.equal(dw, want_dw)


def test_two_calls_at_once():
    """Calls on two streams, each with its own workspace."""
    sets = [layer(t, 512, 256, 8, 2, seed=t) for t in (8, 8, 200, 200)]
    want = [run(*a, 0) for a in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [torch.empty_like(v) for v in want]
    torch.cuda.synchronize()
    for _ in range(5):
        for a, s, o in zip(sets, streams, outs):
            hs.hscale_experts(*a, 0, o, stream=s)
    torch.cuda.synchronize()
    for o, v in zip(outs, want):
        assert torch.equal(o, v)


def test_small_sizes_and_refusals():
    x, ids, w, gate, up, down = layer(3, 64, 32, 4, 2)
    y = torch.full((3, 64), 5.0, dtype=BF16, device=DEV)
    none = (torch.empty(4, 0, 32, dtype=U8, device=DEV), torch.empty(4, 0, 4, dtype=U8, device=DEV), gate[2])
    flat = (torch.empty(4, 64, 0, dtype=U8, device=DEV), torch.empty(4, 64, 0, dtype=U8, device=DEV), gate[2])
    hs.hscale_experts(x, ids, w, none, none, flat, 0, y)
    assert (y == 0).all()
    dw = torch.full((3, 2), 5.0, device=DEV)
    hs.hscale_experts_backward(x, x, ids, w, none, none, flat, 0, y.fill_(5.0), dw)
    assert (y == 0).all() and (dw == 0).all()
    hs.hscale_experts(x[:0], ids[:0], w[:0], gate, up, down, 0, y[:0])
    for bad in (dict(activation=2), dict(ids=ids[:, :1]), dict(gate=up[:2]), dict(y=y[:2]), dict(w=w.double())):
        a = dict(x=x, ids=ids, w=w, gate=gate, up=up, down=down, activation=0, y=y)
        a.update(bad)
        with pytest.raises((TypeError, ValueError, hs.HScaleError)):
            hs.hscale_experts(a["x"], a["ids"], a["w"], a["gate"], a["up"], a["down"], a["activation"], a["y"])
    with pytest.raises(hs.HScaleError):
        hs.hscale_experts(x, ids, w, gate, up, down, 0, y, torch.empty(256, dtype=U8, device=DEV))


def test_a_tokens_bits_do_not_depend_on_its_batch():
    args = layer(900, 448, 208, 5, 2, seed=31)
    x, ids, w, gate, up, down = args
    whole = run(*args, 0)
    for start, count in ((0, 1), (17, 12), (100, 90), (300, 400)):
        part = slice(start, start + count)
        got = run(x[part], ids[part].contiguous(), w[part].contiguous(), gate, up, down, 0)
        assert torch.equal(got, whole[part])
