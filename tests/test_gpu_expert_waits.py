"""Waits of the experts' kernels running out in a block that has several tiles.  In wide tiles (128 slots, 256 in the backward
pass) the unpacking warps take part in the epilogue, and what they owe has to be NaN too, not what an earlier call left in the
workspace; and a warp that gives up must not let the next tile's MMAs overwrite what the others still read.

The library is built once more with one block in which some waits run out at once: of the four epilogue warps for an accumulator (0),
of the unpacking warps (1), or those of a later turn of the ring that these read (2).  Every other wait of the block then
runs out as well, after some milliseconds, and the kernels end normally."""
import concurrent.futures as cf
import ctypes
import subprocess

import pytest
import torch

import paper_2608_28113_gb300 as hs
from paper_2608_28113_gb300 import build as cuda_build
from test_gpu_experts import layer, rows
from test_gpu_failure import both

pytestmark = pytest.mark.gpu
BF16, U8 = torch.bfloat16, torch.uint8
DEV = "cuda"


@pytest.fixture(scope="module", params=[(1, 0), (0, 1), (0, 2), (1, 2)])
def starved_unpacking(request, tmp_path_factory):
    """(block, library): the library with that block's unpacking warps starved."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()
    (block, waits), out = request.param, tmp_path_factory.mktemp("starved_unpacking")

    def obj_of(src):
        if src.stem not in ("experts", "experts_backward"):
            return str(cuda_build.BUILD / (src.stem + ".o"))
        obj = out / (src.stem + ".o")
        subprocess.run([cuda_build.nvcc_path(), *cuda_build.ARCH, *cuda_build.NVCC_FLAGS, f"-DHSCALE_STARVED_BLOCK={block}",
                        f"-DHSCALE_STARVED_WAIT={waits}", "-c", str(src), "-o", str(obj)], check=True, capture_output=True)
        return str(obj)

    with cf.ThreadPoolExecutor(2) as ex:
        objs = list(ex.map(obj_of, cuda_build.sources()))
    so = out / f"libhscale_unpacking{block}{waits}.so"
    subprocess.run([cuda_build.nvcc_path(), *cuda_build.ARCH, "-shared", "-o", str(so), *objs], check=True)
    lib = ctypes.CDLL(str(so))
    for name, (res, args) in hs._SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return block, lib


# tokens: narrow tiles; wide ones, one a block; wide ones, several a block, of as many K blocks that the waits run out
# at the beginning of a tile and inside one
@pytest.mark.parametrize("t, n, inner", [(6, 2048, 2048), (1500, 512, 1024), (9000, 512, 1024), (30000, 256, 384)])
def test_starved_unpacking(starved_unpacking, monkeypatch, t, n, inner):
    count, k = 8, 2
    args = layer(t, n, inner, count, k, seed=12, none=0.0)
    x, ids, w, gate, up, down = args
    dy, _ = rows(t, n, 0, torch.Generator().manual_seed(3))
    ws = torch.empty(hs.hscale_experts_workspace_bytes(t, k, n, inner, count), dtype=U8, device=DEV)
    wsb = torch.empty(hs.hscale_experts_backward_workspace_bytes(t, k, n, inner, count), dtype=U8, device=DEV)

    def forward():
        y = torch.zeros(t, n, dtype=BF16, device=DEV)
        hs.hscale_experts(*args, 0, y, ws)
        return y

    def backward():
        dx, dw = torch.zeros(t, n, dtype=BF16, device=DEV), torch.zeros(t, k, device=DEV)
        hs.hscale_experts_backward(dy, *args, 0, dx, dw, wsb)
        return torch.cat((dx.float(), dw), 1)

    # another call's values, all of them finite, in the workspaces
    other = x.roll(1, 1).contiguous()
    hs.hscale_experts(other, ids, w, gate, up, down, 0, torch.empty_like(other), ws)
    hs.hscale_experts_backward(other, other, ids, w, gate, up, down, 0, torch.empty_like(other), torch.empty_like(w), wsb)
    for call in (forward, backward):
        got, want = both(starved_unpacking, monkeypatch, call)
        lost = got.isnan()
        assert lost.any() and not want.isnan().any()
        assert torch.equal(got[~lost], want[~lost])
