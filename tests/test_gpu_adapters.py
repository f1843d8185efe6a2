"""8-bit checkpoints, and the packed projection with adapters and its gradients, on the GPU, against
their definitions in 64 bits.

Tolerances.  A result is rounded once to bf16: at most 2^-8 of its magnitude.  Before that it is an fp32
sum: on the tensor cores K products enter in K / 16 additions that may each lose a few units of 2^-23 of the
magnitudes summed so far, elsewhere K additions in parallel chains lose less; so K / 4 + 64 units of the sum S of
the terms' magnitudes bound it, for every sum that feeds a result.  Gradients of the adapters take z and dz as pairs of
bf16 numbers, which adds 2^-16 of S.
"""
import zlib

import pytest
import torch

import paper_2608_28113_gb300 as hs

pytestmark = pytest.mark.gpu
BF16, F32, F64, U8, I32 = torch.bfloat16, torch.float32, torch.float64, torch.uint8, torch.int32
DEV = "cuda"
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


def gen(*salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(zlib.crc32(repr(salt).encode()))
    return g


def rows(t, cols, ld, lead=0):
    """bf16 [t, cols] inside a buffer of NaN whose rows are ld long, starting at column lead."""
    return torch.full((t, ld), float("nan"), dtype=BF16, device=DEV)[:, lead:lead + cols]


def ld8(cols, pad=0):
    return (cols + 7) // 8 * 8 + pad


# ---------------------------------------------------------------- 8-bit checkpoints
def e4m3_values(codes):
    return codes.contiguous().view(torch.float8_e4m3fn).to(F64)


def checkpoint64(x, fmt):
    """(values, scale exponents) of the definition, in 64 bits."""
    t, n = x.shape
    full = torch.nn.functional.pad(x.to(F64), (0, -n % 32)).reshape(t, -1, 32)
    amax = full.abs().amax(2)
    mant, exp = torch.frexp(amax)
    e = exp - 7 if fmt == 0 else exp - 9 + (mant > 0.875).to(I32)
    e = torch.where(amax > 0, e, torch.full_like(e, -124)).clamp(min=-124)
    scale = torch.exp2(e.to(F64))[:, :, None]
    v = full / scale
    if fmt == 0:
        q = torch.round(v).clamp(-127, 127)
    else:
        own = torch.frexp(v.abs().clamp(min=2.0 ** -20))[1].to(F64) - 1
        step = torch.exp2(own.clamp(min=-6) - 3)
        q = torch.round(v / step) * step
        q = torch.where(e[:, :, None] == 120, q.clamp(-240, 240), q)  # 256 2^120 is past bf16's range
    return (q * scale).reshape(t, -1)[:, :n], e


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("t, n, pad, lead, ld_c", [
    (1, 1, 0, 0, 1), (1, 31, 0, 0, 31), (3, 32, 0, 0, 32), (5, 33, 8, 0, 40), (7, 200, 0, 3, 200), (300, 1024, 0, 0, 1024),
    (65, 4104, 16, 8, 4104), (2, 28672, 0, 0, 28673)])
def test_checkpoint_round_trip(fmt, t, n, pad, lead, ld_c):
    g = gen("ckpt", fmt, t, n)
    x = rows(t, n, ld8(n, pad + 8), lead)
    x.copy_(torch.randn(t, n, generator=g, device=DEV) * torch.exp2(torch.randint(-30, 30, (t, n), generator=g, device=DEV)))
    x[0, 0] = 0.0
    codes = torch.full((t, ld_c), 77, dtype=U8, device=DEV)[:, :n]
    scales = torch.zeros(t, (n + 31) // 32, dtype=U8, device=DEV)
    hs.hscale_checkpoint_save(x, fmt, codes, scales)
    want, e = checkpoint64(x, fmt)
    assert torch.equal(scales.to(I32), e + 127)
    value = codes.contiguous().view(torch.int8).to(F64) if fmt == 0 else e4m3_values(codes)
    held = value * torch.exp2(e.to(F64)).repeat_interleave(32, dim=1)[:, :n]
    assert torch.equal(held, want)
    out = rows(t, n, ld8(n, 8))
    hs.hscale_checkpoint_load(codes, scales, fmt, out)
    assert torch.equal(out.to(F64), want)
    if ld_c > n:  # nothing beside the rows was written
        assert (codes.as_strided((t, 1), (ld_c, 1), n) == 77).all()


@pytest.mark.parametrize("fmt", [0, 1])
def test_checkpoint_extremes(fmt):
    """Blocks of zeros, of the largest and the smallest magnitudes, of every significand, and with Inf or
    NaN, which spoil their own block only."""
    x = torch.zeros(8, 32, dtype=BF16, device=DEV)
    x[1] = torch.finfo(BF16).max
    x[2] = -torch.finfo(BF16).max
    x[3, :4] = torch.tensor([2.0 ** -133, 2.0 ** -126, -2.0 ** -130, 0.0], device=DEV)
    x[4] = torch.arange(128, 160, device=DEV).to(BF16)
    x[5] = -torch.arange(224, 256, device=DEV).to(BF16)
    x[6, 5] = float("inf")
    x[7, 31] = float("nan")
    codes = torch.empty(8, 32, dtype=U8, device=DEV)
    scales = torch.empty(8, 1, dtype=U8, device=DEV)
    hs.hscale_checkpoint_save(x, fmt, codes, scales)
    out = torch.empty_like(x)
    hs.hscale_checkpoint_load(codes, scales, fmt, out)
    assert torch.equal(out[:6].to(F64), checkpoint64(x[:6], fmt)[0])
    assert out[6:].isnan().all() and (scales[6:] == 255).all()


# ---------------------------------------------------------------- the projection
class Layer:
    """A packed weight, adapters and activations, with their 64-bit results."""

    def __init__(self, t, m, n, count, rank, ids, pad=0, fmt=0, seed=0):
        g = gen("layer", t, m, n, count, rank, seed)
        self.t, self.m, self.n, self.count, self.rank, self.fmt = t, m, n, count, rank, fmt
        self.packed = torch.randint(256, (m, n // 2), generator=g, device=DEV, dtype=U8)
        self.codes = torch.randint(40, 90, (m, n // 16), generator=g, device=DEV, dtype=U8)
        self.sg = torch.rand(1, generator=g, device=DEV) * 1e-3 + 1e-4
        self.x = rows(t, n, ld8(n, pad))
        self.x.copy_(torch.randn(t, n, generator=g, device=DEV))
        self.dy = rows(t, m, ld8(m, pad))
        self.dy.copy_(torch.randn(t, m, generator=g, device=DEV))
        self.a = torch.randn(count, rank, n, generator=g, device=DEV).to(BF16) if count else None
        self.b = torch.randn(count, m, rank, generator=g, device=DEV).to(BF16) if count else None
        self.alpha = torch.rand(count, generator=g, device=DEV) + 0.5 if count else None
        if isinstance(ids, str):
            if ids == "mixed":
                ids = torch.randint(-1, count, (t,), generator=g, device=DEV)
            elif ids == "runs":
                ids = (torch.arange(t, device=DEV) * count) // max(t, 1)
            elif ids == "none":
                ids = torch.full((t,), -1, device=DEV)
            elif ids == "outside":
                ids = torch.randint(-2 ** 31, 2 ** 31, (t,), generator=g, device=DEV)
                ids[::3] = torch.randint(0, count, (ids[::3].numel(),), generator=g, device=DEV)
        self.ids = None if ids is None else ids.to(I32)
        self.which = torch.zeros(t, dtype=torch.int64, device=DEV) if ids is None else ids.to(torch.int64)
        if count == 0:
            self.which = torch.full((t,), -1, dtype=torch.int64, device=DEV)
        self.pad = pad

    def weight(self):
        grid = torch.tensor(GRID + [-v for v in GRID], dtype=F64, device=DEV)
        nib = torch.stack((self.packed & 15, self.packed >> 4), 2).reshape(self.m, self.n)
        scale = e4m3_values(self.codes) * self.sg.to(F64)
        return grid[nib.long()] * scale.repeat_interleave(16, dim=1)

    def members(self):
        return [(a, (self.which == a).nonzero().squeeze(1)) for a in range(self.count)]

    def forward64(self, absolute=False, a=None, b=None, x=None):
        f = (lambda v: v.to(F64).abs()) if absolute else (lambda v: v.to(F64))
        x, a, b = self.x if x is None else x, self.a if a is None else a, self.b if b is None else b
        y = f(x) @ f(self.weight()).T
        for i, on in self.members():
            y[on] += f(self.alpha)[i] * (f(x)[on] @ f(a[i]).T) @ f(b[i]).T
        return y

    def project(self, **kw):
        y = rows(self.t, self.m, ld8(self.m, self.pad))
        hs.hscale_project(self.x, self.packed, self.codes, self.sg, self.a, self.b, self.alpha, self.ids, y, **kw)
        return y

    def checkpoint(self):
        codes = torch.empty(self.t, self.n, dtype=U8, device=DEV)
        scales = torch.empty(self.t, (self.n + 31) // 32, dtype=U8, device=DEV)
        hs.hscale_checkpoint_save(self.x, self.fmt, codes, scales)
        held = torch.empty(self.t, self.n, dtype=BF16, device=DEV)
        hs.hscale_checkpoint_load(codes, scales, self.fmt, held)
        return codes, scales, held

    def backward(self, want=("dx", "da", "db"), **kw):
        codes, scales, held = self.checkpoint()
        dx = rows(self.t, self.n, ld8(self.n, self.pad)) if "dx" in want else None
        da = torch.full_like(self.a, float("nan")) if "da" in want and self.count else None
        db = torch.full_like(self.b, float("nan")) if "db" in want and self.count else None
        hs.hscale_project_backward(self.dy, codes, scales, self.fmt, self.packed, self.codes, self.sg, self.a, self.b,
                                   self.alpha, self.ids, dx, da, db, **kw)
        return dx, da, db, held

    def backward64(self, held, absolute=False):
        f = (lambda v: v.to(F64).abs()) if absolute else (lambda v: v.to(F64))
        dy, x = f(self.dy), f(held)
        dx = dy @ f(self.weight())
        da = db = None
        if self.count:
            da, db = torch.zeros_like(self.a, dtype=F64), torch.zeros_like(self.b, dtype=F64)
        for i, on in self.members():
            dz = f(self.alpha)[i] * dy[on] @ f(self.b[i])
            dx[on] += dz @ f(self.a[i])
            da[i] = dz.T @ x[on]
            db[i] = f(self.alpha)[i] * dy[on].T @ (x[on] @ f(self.a[i]).T)
        return dx, da, db


def check(got, want, magnitude, depth, extra=0.0):
    err = (got.to(F64) - want).abs()
    tol = want.abs() * 2.0 ** -8 + magnitude * ((depth / 4 + 64) * 2.0 ** -23 + extra) + 2.0 ** -133
    worst = (err / tol).max().item() if err.numel() else 0.0
    assert worst <= 1.0 and not got.isnan().any(), worst


FORWARD = [
    # t, m, n, adapters, rank, ids, pad
    (1, 1, 16, 1, 8, None, 0), (1, 24, 64, 2, 16, "mixed", 0), (1, 4096, 1024, 8, 16, "mixed", 0),
    (2, 129, 48, 3, 8, "mixed", 8), (7, 100, 2000, 3, 24, "outside", 16), (8, 512, 8192, 8, 16, "mixed", 0),
    (9, 257, 528, 9, 64, "mixed", 0), (15, 3001, 256, 4, 128, "runs", 0), (16, 1000, 4096, 16, 32, "mixed", 0),
    (17, 130, 1040, 2, 8, "none", 0), (31, 64, 160, 3, 16, "mixed", 0), (33, 333, 336, 33, 40, "mixed", 24),
    (64, 640, 1024, 64, 16, "mixed", 0), (65, 1, 2064, 2, 16, "runs", 0), (100, 127, 128, 1, 16, None, 0),
    (127, 128, 64, 5, 32, "runs", 0), (129, 385, 80, 2, 16, "mixed", 8), (200, 300, 400, 0, 0, None, 0),
    (256, 256, 512, 7, 16, "runs", 0), (257, 1025, 1024, 3, 64, "runs", 0), (513, 200, 272, 300, 8, "mixed", 0),
    (1000, 640, 704, 4, 16, "runs", 0), (2000, 1111, 528, 2, 16, "outside", 0), (1, 28672, 16, 1, 8, None, 0),
    (4, 16, 28672, 2, 8, "mixed", 0), (40, 48, 14336, 4, 16, "mixed", 0), (5, 70, 112, 0, 0, None, 0)]


@pytest.mark.parametrize("t, m, n, count, rank, ids, pad", FORWARD)
def test_project(t, m, n, count, rank, ids, pad):
    L = Layer(t, m, n, count, rank, ids, pad)
    y = L.project()
    check(y, L.forward64(), L.forward64(absolute=True), n + rank)
    # the same bits again, and nothing beside the rows
    assert torch.equal(L.project(), y)
    if y.stride(0) > m and t > 1:
        assert y.as_strided((t, y.stride(0) - m), (y.stride(0), 1), m)[:-1].isnan().all()


BACKWARD = [
    (1, 1, 16, 1, 8, None, 0, 0), (1, 64, 48, 2, 16, "mixed", 0, 1), (7, 130, 2000, 3, 24, "outside", 16, 0),
    (16, 1000, 416, 16, 32, "mixed", 0, 1), (33, 333, 336, 33, 40, "mixed", 24, 0), (64, 64, 1024, 2, 128, "runs", 0, 0),
    (65, 1, 2064, 2, 16, "runs", 0, 1), (96, 512, 1024, 2, 16, "runs", 8, 0), (129, 385, 80, 2, 16, "mixed", 8, 0),
    (200, 300, 400, 0, 0, None, 0, 0), (257, 1025, 1024, 3, 64, "runs", 0, 1), (513, 200, 272, 300, 8, "mixed", 0, 0),
    (700, 264, 528, 4, 16, "none", 0, 0), (1000, 640, 704, 1, 16, None, 0, 1), (3000, 129, 176, 5, 48, "mixed", 0, 0),
    (9000, 72, 96, 2, 16, "runs", 0, 0), (20, 2064, 64, 2, 8, "mixed", 0, 0)]


@pytest.mark.parametrize("t, m, n, count, rank, ids, pad, fmt", BACKWARD)
def test_backward(t, m, n, count, rank, ids, pad, fmt):
    L = Layer(t, m, n, count, rank, ids, pad, fmt)
    dx, da, db, held = L.backward()
    wx, wa, wb = L.backward64(held)
    sx, sa, sb = L.backward64(held, absolute=True)
    check(dx, wx, sx, 2 * m + rank)
    if count:
        check(da, wa, sa, t + m, 2.0 ** -16)
        check(db, wb, sb, t + n, 2.0 ** -16)
        for i, on in L.members():
            if on.numel() == 0:
                assert (da[i] == 0).all() and (db[i] == 0).all()
    again = L.backward()
    assert torch.equal(again[0], dx) and (not count or (torch.equal(again[1], da) and torch.equal(again[2], db)))


@pytest.mark.parametrize("want", [("dx",), ("da",), ("db",), ("da", "db"), ()])
def test_backward_in_parts(want):
    L = Layer(50, 72, 96, 3, 16, "mixed")
    whole = dict(zip(("dx", "da", "db"), L.backward()))
    part = dict(zip(("dx", "da", "db"), L.backward(want)))
    for name in ("dx", "da", "db"):
        assert (part[name] is None) == (name not in want)
        if name in want:
            assert torch.equal(part[name], whole[name])


def test_backward_against_differences():
    """The loss <c, y> is linear in A and in B alone and in x: central differences of the 64-bit forward
    are exact, and dy = c."""
    L = Layer(40, 56, 64, 3, 8, "mixed")
    dx, da, db, held = L.backward()
    c, g = L.dy.to(F64), gen("differences")
    sx, sa, sb = L.backward64(held, absolute=True)

    def loss(**kw):
        return (c * L.forward64(x=kw.pop("x", held.to(F64)), **kw)).sum()

    for name, grad, mag, depth in (("x", dx, sx, 2 * 56), ("a", da, sa, 96), ("b", db, sb, 104)):
        base = held.to(F64) if name == "x" else getattr(L, name).to(F64)
        v = torch.randn(base.shape, generator=g, device=DEV, dtype=F64)
        slope = (loss(**{name: base + v}) - loss(**{name: base - v})) / 2
        tol = (v.abs() * (grad.to(F64).abs() * 2.0 ** -8 + mag * ((depth / 4 + 64) * 2.0 ** -23 + 2.0 ** -16))).sum()
        assert (slope - (v * grad.to(F64)).sum()).abs() <= tol


@pytest.mark.parametrize("t", [16, 64, 300])
def test_every_weight_value_is_exact(t):
    """x of unit rows reads W_hat itself: every code and nibble, with s_g a power of two."""
    m, n = 126, 256
    L = Layer(t, m, n, 0, 0, None)
    L.sg.fill_(0.25)
    L.codes = torch.arange(1, 127, device=DEV, dtype=U8)[:, None].expand(m, n // 16).contiguous()
    nib = torch.arange(n, device=DEV) % 16
    L.packed = ((nib[1::2] << 4) | nib[0::2]).to(U8)[None].expand(m, n // 2).contiguous()
    L.x.zero_()
    cols = (torch.arange(t, device=DEV) * 37) % n
    L.x[torch.arange(t, device=DEV), cols] = 2.0
    assert torch.equal(L.project().to(F64), 2.0 * L.weight().T[cols])
    dy = rows(m, m, ld8(m))
    dy.copy_(torch.eye(m, device=DEV))
    dx = rows(m, n, n)
    hs.hscale_project_backward(dy, None, None, 0, L.packed, L.codes, L.sg, None, None, None, None, dx, None, None)
    assert torch.equal(dx.to(F64), L.weight())


def test_codes_off_the_ladder_are_read_as_everywhere():
    L = Layer(20, 40, 64, 0, 0, None)
    L.codes[0], L.codes[1], L.codes[2] = 0, 127, 200
    got = L.project()
    L.codes[0], L.codes[1], L.codes[2] = 1, 126, 72
    assert torch.equal(got, L.project())


@pytest.mark.parametrize("t", [3, 16, 40, 300])
def test_inf_and_nan_stay_in_their_token_and_adapter(t):
    L = Layer(t, 200, 512, 4, 16, "mixed", seed=1)
    L.ids[0], L.ids[1], L.ids[2] = 0, 1, 2
    L.ids[3:][L.ids[3:] == 1] = 3  # token 1 alone uses adapter 1
    L.which = L.ids.long()
    clean, clean_b = L.project(), L.backward()
    L.a[1, 3, 100], L.b[1, 7, 2] = float("inf"), float("nan")
    L.x[0, 5] = float("nan")
    y = L.project()
    others = torch.arange(t, device=DEV) >= 2
    assert torch.equal(y[others], clean[others])
    assert y[0].isnan().all() and y[1].isnan().any()
    dx, da, db, _ = L.backward()
    assert torch.equal(dx[others], clean_b[0][others]) and torch.equal(dx[0], clean_b[0][0])
    assert dx[1].isnan().any()
    for i in (2, 3):
        assert torch.equal(da[i], clean_b[1][i]) and torch.equal(db[i], clean_b[2][i])
    L.dy[2, 9] = float("inf")
    dx, da, db, _ = L.backward()
    others = torch.arange(t, device=DEV) >= 3
    assert torch.equal(dx[others], clean_b[0][others])
    assert torch.equal(da[3], clean_b[1][3]) and torch.equal(db[3], clean_b[2][3])


@pytest.mark.parametrize("t, m, n, rank, order", [
    (64, 200, 512, 16, "mixed"), (300, 200, 512, 16, "mixed"), (300, 264, 272, 64, "mixed"), (700, 130, 400, 8, "runs"),
    (257, 640, 2048, 24, "runs"), (2000, 384, 256, 40, "mixed")])
def test_a_broken_adapter_of_many_tokens(t, m, n, rank, order):
    """One of three adapters holds an Inf and a NaN: the others' tokens keep their bits, its own tokens keep
    theirs at the outputs that its factors do not spoil."""
    L = Layer(t, m, n, 3, rank, order, seed=2)
    clean, clean_b = L.project(), L.backward()
    on = L.which == 1
    L.b[1, 7, 2], L.b[1, m - 1, rank - 1] = float("nan"), float("inf")
    y = L.project()
    assert torch.equal(y[~on], clean[~on])
    spoilt = torch.zeros(m, dtype=torch.bool, device=DEV)
    spoilt[[7, m - 1]] = True
    assert torch.equal(y[on][:, ~spoilt], clean[on][:, ~spoilt])
    assert y[on][:, 7].isnan().all() and not y[on][:, m - 1].isfinite().any()
    L.b[1] = Layer(t, m, n, 3, rank, order, seed=2).b[1]
    L.a[1, rank - 1, 9], L.a[1, 0, n - 2] = float("-inf"), float("nan")
    dx, da, db, _ = L.backward()
    assert torch.equal(dx[~on], clean_b[0][~on])
    spoilt = torch.zeros(n, dtype=torch.bool, device=DEV)
    spoilt[[9, n - 2]] = True
    assert torch.equal(dx[on][:, ~spoilt], clean_b[0][on][:, ~spoilt])
    assert not dx[on][:, spoilt].isfinite().any()
    assert torch.equal(da, clean_b[1])  # z alone depends on A
    assert torch.equal(db[[0, 2]], clean_b[2][[0, 2]])


def test_another_stream_and_a_given_workspace():
    L = Layer(70, 300, 512, 5, 16, "mixed")
    want, wantb = L.project(), L.backward()
    side = torch.cuda.Stream()
    ws = torch.full((hs.hscale_project_workspace_bytes(70, 300, 512, 5, 16),), 255, dtype=U8, device=DEV)
    wsb = torch.full((hs.hscale_project_backward_workspace_bytes(70, 300, 512, 5, 16),), 255, dtype=U8, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, gotb = L.project(workspace=ws), L.backward(workspace=wsb)
    side.synchronize()
    assert torch.equal(got, want) and all(torch.equal(p, q) for p, q in zip(gotb, wantb))
    with pytest.raises(hs.HScaleError):
        L.project(workspace=ws[:256])


@pytest.mark.parametrize("t, m", [(1, 4096), (12, 640), (48, 640), (300, 640)])
def test_replayed_from_a_graph(t, m):
    L = Layer(t, m, 1024, 3, 16, "mixed")
    ws = torch.empty(hs.hscale_project_backward_workspace_bytes(t, m, 1024, 3, 16), dtype=U8, device=DEV)
    want, wantb = L.project(workspace=ws), L.backward(workspace=ws)
    y = rows(t, m, ld8(m))
    dx, da, db = (torch.zeros_like(v) for v in wantb[:3])
    codes, scales, _ = L.checkpoint()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hs.hscale_project(L.x, L.packed, L.codes, L.sg, L.a, L.b, L.alpha, L.ids, y, ws)
        hs.hscale_project_backward(L.dy, codes, scales, 0, L.packed, L.codes, L.sg, L.a, L.b, L.alpha, L.ids, dx, da, db, ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    assert torch.equal(dx, wantb[0]) and torch.equal(da, wantb[1]) and torch.equal(db, wantb[2])


def test_empty_sums():
    """Zero tokens and zero widths: outputs that exist are zero, and nothing else is touched."""
    L = Layer(6, 40, 64, 2, 8, "mixed")
    da, db = torch.ones_like(L.a), torch.ones_like(L.b)
    none = torch.empty(0, 64, dtype=U8, device=DEV)
    hs.hscale_project_backward(L.dy[:0], none, none[:, :2], 0, L.packed, L.codes, L.sg, L.a, L.b, L.alpha, L.ids[:0],
                               torch.empty(0, 64, dtype=BF16, device=DEV), da, db)
    assert (da == 0).all() and (db == 0).all()
    y = torch.ones(6, 40, dtype=BF16, device=DEV)
    hs.hscale_project(torch.empty(6, 0, dtype=BF16, device=DEV), L.packed[:, :0].contiguous(), L.codes[:, :0].contiguous(), L.sg, None,
                      None, None, None, y)
    assert (y == 0).all()
    hs.hscale_project(L.x[:0], L.packed, L.codes, L.sg, L.a, L.b, L.alpha, L.ids[:0], y[:0])
    dx = torch.ones(6, 64, dtype=BF16, device=DEV)
    hs.hscale_project_backward(L.dy[:, :0], None, None, 0, L.packed[:0], L.codes[:0], L.sg, None, None, None, None, dx, None,
                               None)
    assert (dx == 0).all()


def test_binding_refusals():
    L = Layer(4, 24, 64, 2, 8, "mixed")
    y = rows(4, 24, 24)
    bad = torch.zeros(1, dtype=I32, device=DEV)
    for args in ((L.x, L.packed[:, 1:], L.codes, L.sg, L.a, L.b, L.alpha, L.ids, y),
                 (L.x, L.packed, L.codes, L.sg, L.a, L.b[:1], L.alpha, L.ids, y),
                 (L.x, L.packed, L.codes, L.sg, L.a, L.b, L.alpha, bad, y),
                 (L.x, L.packed, L.codes, L.sg, None, L.b, L.alpha, L.ids, y),
                 (L.x.T, L.packed, L.codes, L.sg, L.a, L.b, L.alpha, L.ids, y)):
        with pytest.raises(ValueError):
            hs.hscale_project(*args)
    with pytest.raises(TypeError):
        hs.hscale_project(L.x, L.packed, L.codes, L.sg, L.a, L.b, L.alpha, L.ids.long(), y)
    with pytest.raises(hs.HScaleError):  # rows off the 16-byte grid
        hs.hscale_project(rows(4, 64, 80, 1), L.packed, L.codes, L.sg, L.a, L.b, L.alpha, L.ids, y)
    assert hs.hscale_device_error_flags() == 0
