"""What the build compiles of the router is what its calls launch."""
import re

import pytest

from paper_2608_28113_gb300 import build


def test_router_kernels_are_the_launched_ones():
    build.build()
    log = build.BUILD / "ptxas.log"
    if not log.exists():
        pytest.skip("built elsewhere")
    names = set(re.findall(r"Compiling entry function '\w*?\d+(route\w*_kernelI\w*?Li\d+)E", log.read_text()))
    bf16, sizes = "I13__nv_bfloat16Li", (1, 2, 4, 8, 32)
    # up to 256 bf16 logits as sorted words; all others, and the gradient, by type and size
    want = {f"route_words_kernelILi{s}" for s in sizes[:4]} | {f"route_kernel{bf16}32"} | {f"route_kernelIfLi{s}" for s in sizes}
    want |= {f"route_backward_kernel{t}{s}" for t in ("IfLi", bf16) for s in sizes}
    assert names == want
