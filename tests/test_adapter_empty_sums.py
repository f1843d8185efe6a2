"""The backward pass of a projection without outputs (m == 0), on the CPU: pointers of empty matrices may be null, and
a call with nothing to write does nothing."""
import pytest

import paper_2608_28113_gb300 as hs
from paper_2608_28113_gb300 import build

OK, ERR_NULL, ERR_SHAPE, ERR_ALIGN, ERR_ARG = range(5)
P = 4096  # an aligned address that no call here touches


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hs.load()


# db has no elements, and dx and da are not wanted
EMPTY = dict(dy=None, tokens=4, m=0, ld_dy=0, xc=P, ld_xc=64, xs=P, ld_xs=2, fmt=0, n=64, packed=None, codes=None, sg=None,
             a=P, b=None, alpha=P, adapters=2, rank=16, of=P, dx=None, ld_dx=0, da=None, db=P, ws=None, ws_bytes=0, stream=None)


@pytest.mark.parametrize("change, status", [
    ({}, OK), (dict(dy=P), OK), (dict(xc=None, xs=None), OK), (dict(dy=P + 1), OK), (dict(fmt=2), ERR_ARG), (dict(ld_xc=63), ERR_SHAPE),
    (dict(ld_xs=1), ERR_SHAPE), (dict(db=P + 8), ERR_ALIGN)])
def test_no_outputs(lib, change, status):
    assert lib.hscale_project_backward(*{**EMPTY, **change}.values()) == status
