"""A call on a given stream that allocates its own workspace takes that stream's memory: the allocator hands the memory of
another stream to that one's next allocation as soon as the call returns, with the call's kernels still to run."""
import pytest
import torch

import paper_2608_28113_gb300 as hs
from test_gpu_adapters import BF16, DEV, I32, U8, Layer, gen, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


def held_by(stream):
    """Bytes of the allocator's segments that belong to a stream."""
    return sum(s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == stream.cuda_stream)


def project(how):
    L = Layer(3000, 136, 272, 3, 64, "mixed")
    y, need = rows(3000, 136, 136), hs.hscale_project_workspace_bytes(3000, 136, 272, 3, 64)
    return need, (y,), lambda: hs.hscale_project(L.x, L.packed, L.codes, L.sg, L.a, L.b, L.alpha, L.ids, y, **how())


def backward(how):
    L = Layer(3000, 136, 272, 3, 64, "mixed")
    codes, scales, _ = L.checkpoint()
    dx, da, db = rows(3000, 272, 272), torch.empty_like(L.a), torch.empty_like(L.b)
    need = hs.hscale_project_backward_workspace_bytes(3000, 136, 272, 3, 64)
    return need, (dx, da, db), lambda: hs.hscale_project_backward(L.dy, codes, scales, 0, L.packed, L.codes, L.sg, L.a, L.b,
                                                                  L.alpha, L.ids, dx, da, db, **how())


def hessian(how):
    x = torch.randn(3000, 521, generator=gen("stream h"), device=DEV).to(BF16)[:, 1:]
    H = torch.empty(520, 520, device=DEV)

    def call():
        hs.hscale_hessian_full_accumulate(x, H, **how())

    return hs.hscale_hessian_full_workspace_bytes(3000, 520), (H,), call


def factor(how):
    x = torch.randn(600, 512, generator=gen("stream f"), device=DEV)
    H, U, info = (x.T @ x).contiguous(), torch.empty(512, 512, device=DEV), torch.empty(3, dtype=I32, device=DEV)
    return hs.hscale_gptq_factor_workspace_bytes(512), (U, info), lambda: hs.hscale_gptq_factor(H, 0.01, U, None, info, **how())


def gptq(how):
    m, n = 256, 512
    w = (torch.randn(m, n, generator=gen("stream g"), device=DEV) * 0.02).to(BF16)
    U = torch.eye(n, device=DEV) + torch.triu(torch.randn(n, n, generator=gen("stream u"), device=DEV) * 0.01, 1)
    h, sg = torch.ones(n, device=DEV), w.float().abs().max().reshape(1) / 2688
    codes, packed = torch.empty(m, n // 16, dtype=U8, device=DEV), torch.empty(m, n // 2, dtype=U8, device=DEV)
    return hs.hscale_gptq_workspace_bytes(m, n, 128), (codes, packed), lambda: hs.hscale_gptq_hscale(
        w, U, h, sg, None, 128, 2, 2, codes, packed, **how())


@pytest.mark.parametrize("handle", ["stream", "number"])
@pytest.mark.parametrize("make", [project, backward, hessian, factor, gptq])
def test_the_workspace_is_the_streams(make, handle):
    given = {}
    need, outs, call = make(lambda: given)
    torch.cuda.synchronize()
    for out in outs:
        out.zero_()
    call()  # the current stream, whose memory the workspace is
    want = [out.clone() for out in outs]
    for out in outs:
        out.zero_()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = held_by(side)
    given["stream"] = side if handle == "stream" else side.cuda_stream
    call()
    assert held_by(side) >= before + need > before
    assert torch.cuda.current_stream() != side
    side.synchronize()
    assert all(torch.equal(out, ref) for out, ref in zip(outs, want))


@pytest.mark.parametrize("default", [0, 1])
def test_the_default_streams_numbers(default):
    given = {}
    _, (y,), call = project(lambda: given)
    call()
    want = y.clone()
    y.zero_()
    given["stream"] = default
    call()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
