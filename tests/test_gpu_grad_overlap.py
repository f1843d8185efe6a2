"""hscale_grad_clip onto its own tensors, beside them, and what it refuses, through the binding."""
import pytest
import torch

import paper_2608_28113_gb300 as hs

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    hs.load()


def test_places_that_do_not_overlap():
    room = torch.ones(4096, device=DEV)
    a, b, c, d = room[:1000], room[1000:1001], room[1001:1001], room[3000:]
    norm = torch.empty(1, device=DEV)
    want = torch.full((1000,), 0.5, device=DEV)
    # onto its own, right behind another's, an empty one anywhere
    hs.hscale_grad_clip([a, d, c, b], 0.5 * 2097 ** 0.5, norm, [a, room[1001:2097], room[500:500], b])
    assert (room[:1000] - want).abs().max() < 1e-6 and (room[1000:2097] - 0.5).abs().max() < 1e-6
    assert (room[2097:] == 1.0).all()
    # the same gradient read twice, written to two places
    one, out = torch.ones(64, device=DEV), torch.zeros(2, 64, device=DEV)
    hs.hscale_grad_clip([one, one], 0.5 * 128 ** 0.5, norm, [out[0], out[1]])
    assert (out - 0.5).abs().max() < 1e-6 and (one == 1.0).all()
    # in place, in any order
    parts = list(torch.ones(100, 50, device=DEV).unbind(0))
    hs.hscale_grad_clip(parts[::-1], 0.5 * 5000 ** 0.5, norm)
    assert all((p - 0.5).abs().max() < 1e-6 for p in parts)


def test_overlaps_are_refused():
    room = torch.ones(64, device=DEV)
    norm = torch.empty(1, device=DEV)
    a, b = room[:16], room[16:32]
    before = room.clone()
    for tensors, out in (([a, b], [b, a]), ([a, b], [b, room[32:48]]), ([a], [room[8:24]]), ([a, b], [a, room[15:31]]),
                         ([a, a], [a, room[32:48]])):
        with pytest.raises((ValueError, hs.HScaleError)):
            hs.hscale_grad_clip(tensors, 1.0, norm, out)
        with pytest.raises((ValueError, hs.HScaleError)):
            hs.hscale_grad_clip(hs.hscale_tensors(tensors), 1.0, norm, hs.hscale_tensors(out))
    torch.cuda.synchronize()
    assert torch.equal(room, before)
