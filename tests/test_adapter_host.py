"""The adapter operators' refusals, on the CPU: nothing is enqueued for a bad argument."""
import pytest
import torch

import paper_2608_28113_gb300 as hs
from paper_2608_28113_gb300 import build

OK, ERR_NULL, ERR_SHAPE, ERR_ALIGN, ERR_ARG, ERR_CUDA, ERR_WS = range(7)
P = 4096  # an aligned address that no refused call touches


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hs.load()


SAVE = dict(x=P, tokens=4, n=48, ld_x=48, fmt=0, codes=P, ld_codes=48, scales=P, ld_scales=2, stream=None)


@pytest.mark.parametrize("change, status", [
    (dict(fmt=2), ERR_ARG), (dict(fmt=-1), ERR_ARG), (dict(tokens=-1), ERR_SHAPE), (dict(n=-1), ERR_SHAPE),
    (dict(ld_x=47), ERR_SHAPE), (dict(ld_codes=47), ERR_SHAPE), (dict(ld_scales=1), ERR_SHAPE),
    (dict(x=None), ERR_NULL), (dict(codes=None), ERR_NULL), (dict(scales=None), ERR_NULL), (dict(x=P + 1), ERR_ALIGN),
    (dict(tokens=1 << 31), ERR_SHAPE), (dict(tokens=1 << 30, ld_x=1 << 40), ERR_SHAPE),
    (dict(tokens=0, x=None), OK), (dict(n=0, codes=None), OK)])
def test_checkpoint_refusals(lib, change, status):
    a = {**SAVE, **change}
    assert lib.hscale_checkpoint_save(*a.values()) == status
    assert lib.hscale_checkpoint_load(a["codes"], a["ld_codes"], a["scales"], a["ld_scales"], a["tokens"], a["n"],
                                      a["fmt"], a["x"], a["ld_x"], None) == status


PROJECT = dict(x=P, tokens=4, n=64, ld_x=64, packed=P, codes=P, sg=P, m=24, a=P, b=P, alpha=P, adapters=2, rank=16,
               of=P, y=P, ld_y=24, ws=P, ws_bytes=1 << 20, stream=None)
SHARED = [
    (dict(tokens=-1), ERR_SHAPE), (dict(m=-1), ERR_SHAPE), (dict(n=72, ld_x=72, ld_dx=72, ld_xc=72), ERR_SHAPE),
    (dict(adapters=-1), ERR_SHAPE), (dict(adapters=65536), ERR_SHAPE), (dict(rank=0), ERR_SHAPE),
    (dict(rank=12), ERR_SHAPE), (dict(rank=136), ERR_SHAPE), (dict(packed=None), ERR_NULL),
    (dict(codes=None), ERR_NULL), (dict(sg=None), ERR_NULL), (dict(a=None), ERR_NULL), (dict(b=None), ERR_NULL),
    (dict(alpha=None), ERR_NULL), (dict(packed=P + 4), ERR_ALIGN), (dict(a=P + 8), ERR_ALIGN),
    (dict(b=P + 2), ERR_ALIGN), (dict(of=P + 2), ERR_ALIGN), (dict(ws=None), ERR_WS), (dict(ws_bytes=255), ERR_WS),
    (dict(ws=P + 16), ERR_WS)]


@pytest.mark.parametrize("change, status", SHARED + [
    (dict(ld_x=56), ERR_SHAPE), (dict(ld_y=16), ERR_SHAPE), (dict(ld_x=68), ERR_ALIGN), (dict(ld_y=28), ERR_ALIGN),
    (dict(x=None), ERR_NULL), (dict(y=None), ERR_NULL), (dict(x=P + 2), ERR_ALIGN), (dict(y=P + 8), ERR_ALIGN),
    (dict(tokens=0, x=None, y=None, ws=None), OK), (dict(m=0, y=None, ws=None), OK)])
def test_project_refusals(lib, change, status):
    a = {**PROJECT, **{k: v for k, v in change.items() if k in PROJECT}}
    assert lib.hscale_project(*a.values()) == status


BACKWARD = dict(dy=P, tokens=4, m=24, ld_dy=24, xc=P, ld_xc=64, xs=P, ld_xs=2, fmt=0, n=64, packed=P, codes=P, sg=P, a=P,
                b=P, alpha=P, adapters=2, rank=16, of=P, dx=P, ld_dx=64, da=P, db=P, ws=P, ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("change, status", SHARED + [
    (dict(ld_dy=16), ERR_SHAPE), (dict(ld_dx=56), ERR_SHAPE), (dict(ld_xc=63), ERR_SHAPE), (dict(ld_xs=1), ERR_SHAPE),
    (dict(fmt=7), ERR_ARG), (dict(dy=None), ERR_NULL), (dict(xc=None), ERR_NULL), (dict(xs=None), ERR_NULL),
    (dict(dy=P + 2), ERR_ALIGN), (dict(dx=P + 2), ERR_ALIGN), (dict(da=P + 8), ERR_ALIGN), (dict(db=P + 8), ERR_ALIGN),
    (dict(tokens=0, dy=None, dx=None, da=None, db=None), OK)])
def test_backward_refusals(lib, change, status):
    a = {**BACKWARD, **{k: v for k, v in change.items() if k in BACKWARD}}
    assert lib.hscale_project_backward(*a.values()) == status


def test_workspace_queries(lib):
    assert hs.hscale_project_workspace_bytes(0, 64, 64, 1, 16) == 0
    assert hs.hscale_project_workspace_bytes(5, 64, 64, 0, 0) == 0
    assert hs.hscale_project_workspace_bytes(5, 64, 64, 1, 16) >= 5 * 16 * 4
    assert hs.hscale_project_backward_workspace_bytes(5, 64, 64, 1, 16) >= 2 * 5 * 16 * 4
    big = 1 << 40  # no overflow into a small number
    assert hs.hscale_project_workspace_bytes(big, 64, 64, 1, 128) >= big


def test_binding_refuses_what_it_cannot_marshal(lib):
    x = torch.zeros(2, 32, dtype=torch.bfloat16)
    u8 = torch.zeros(2, 32, dtype=torch.uint8)
    with pytest.raises(TypeError):
        hs.hscale_checkpoint_save(x, 0, u8, u8)
    with pytest.raises(ValueError):
        hs.hscale_checkpoint_load(u8, u8, 0, x[0])
    with pytest.raises(TypeError):
        hs.hscale_project(x, u8, u8, x, None, None, None, None, x)
    with pytest.raises(ValueError):
        hs.hscale_project(x[0], u8, u8, x, None, None, None, None, x)
    with pytest.raises(ValueError):
        hs.hscale_project_backward(x[0], u8, u8, 0, u8, u8, x, None, None, None, None, x, None, None)
