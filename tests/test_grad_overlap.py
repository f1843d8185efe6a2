"""What hscale_grad_clip writes overlaps nothing else that it reads or writes: refused on the host, whichever way it is called."""
import ctypes

import pytest

import paper_2608_28113_gb300 as hs
from paper_2608_28113_gb300 import build

OK, ERR_NULL, ERR_SHAPE, ERR_ALIGN, ERR_ARG, ERR_CUDA, ERR_WS = range(7)
P = 1 << 20
BF16, F32, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def clip():
    build.build()
    lib = hs.load()

    def call(tensors, out, types=None, ws=P, norm=P // 2):
        """tensors: (address, elements) of each; out: addresses, or None."""
        def array(kind, v):
            return None if v is None else (kind * len(v))(*v)
        return lib.hscale_grad_clip(array(ctypes.c_void_p, [p for p, _ in tensors]), array(ctypes.c_int64, [n for _, n in tensors]),
                                    array(ctypes.c_int32, types or [F32] * len(tensors)), len(tensors), 1.0, norm,
                                    array(ctypes.c_void_p, out), ws, 1 << 20, None)
    return call


# addresses of tensors of 256 fp32 elements, 1024 bytes
A, B, C = P, P + 1024, P + 2048


@pytest.mark.parametrize("tensors, out", [
    ([(A, 256), (A, 256)], None),                                     # written twice
    ([(A, 256), (A + 1020, 256)], None),                              # one element of both
    ([(B, 256), (C, 256), (A, 257)], None),                           # behind another in the list
    ([(A, 256), (B, 256)], [C, C]),                                   # one place for both
    ([(A, 256), (B, 256)], [C, C + 1020]),
    ([(A, 256), (B, 256)], [B, C]),                                   # onto the other's input
    ([(A, 256), (B, 256)], [B, A]),                                   # exchanged
    ([(A, 256), (B, 256)], [A, B - 4]),                               # onto its own in part, and the other's
    ([(A, 256)], [A + 4]),                                            # onto its own in part
    ([(A, 256), (C, 256)], [A, A + 1020]),
    ([(A, 256), (A, 256)], [A, C]),                                   # its own, which another is too
    ([(A, 256), (A + 512, 16)], [A, C]),
    ([(C, 16)] * 3 + [(A, 256)], [P + 8192, P + 9216, P + 10240, C + 60]),
    ([(P + 4096 * i, 1024) for i in range(2000)] + [(P + 4096 * 777 + 4092, 1)], None),
    ([(P + 4096 * i, 1024) for i in range(2000)], [P + 4096 * (i + 1999) for i in range(2000)]),
])
def test_overlaps_are_refused(clip, tensors, out):
    assert clip(tensors, out) == ERR_ARG
    assert clip(tensors[::-1], out[::-1] if out else None) == ERR_ARG


@pytest.mark.parametrize("norm", [A, A + 512, A + 1020, B + 1020, P + 8192, P + 8192 + 2044])
def test_the_norm_is_written_too(clip, norm):
    assert clip([(A, 256), (B, 256)], [P + 8192, P + 8192 + 1024], norm=norm) == ERR_ARG
    if norm < P + 8192:
        assert clip([(A, 256), (B, 256)], None, norm=norm) == ERR_ARG


def test_sizes_go_by_the_type(clip):
    assert clip([(A, 256), (A + 512, 256)], None, [F32, F32]) == ERR_ARG
    assert clip([(A, 256), (A + 510, 256)], None, [BF16, F16]) == ERR_ARG
    # what is refused for another reason is refused for that
    assert clip([(A, 256), (A, 256)], None, ws=None) == ERR_WS
    assert clip([(A, 256), (A, 256)], [C, None]) == ERR_NULL
    assert clip([(A, 256), (A, -1)], [C, C]) == ERR_SHAPE


def test_the_refusal_says_so(clip):
    with pytest.raises(hs.HScaleError, match="overlap"):
        hs._check("hscale_grad_clip", clip([(A, 256), (A, 256)], None))
