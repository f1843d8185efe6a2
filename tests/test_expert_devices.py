"""Tensors of one call on different devices, or on another than the current one: refused by the binding, on the CPU with
tensors that only say where they are."""
import pytest
import torch

import paper_2608_28113_gb300 as hs

BF16, F32, U8, I32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32


class On(torch.Tensor):
    """A CPU tensor that says that it is on a GPU."""
    is_cuda = True
    where = 0

    def get_device(self):
        return self.where


def on(where, *shape, dtype):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(On)
    t.where = where
    return t


@pytest.fixture(autouse=True)
def no_gpu(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *args: 0
            raise AssertionError(f"{name} was called")

    monkeypatch.setattr(hs, "_lib", Library())
    monkeypatch.setattr(hs, "load", lambda: hs._lib)


def layer(**elsewhere):
    at = lambda name: elsewhere.get(name, elsewhere.get("all", 0))  # noqa: E731
    t, n, inner, count, k = 3, 32, 16, 4, 2
    a = dict(dy=on(at("dy"), t, n, dtype=BF16), x=on(at("x"), t, n, dtype=BF16), y=on(at("y"), t, n, dtype=BF16),
             ids=on(at("ids"), t, k, dtype=I32), weights=on(at("weights"), t, k, dtype=F32),
             dweights=on(at("dweights"), t, k, dtype=F32), ws=on(at("ws"), 4096, dtype=U8))
    for m, rows, cols in (("gate", inner, n), ("up", inner, n), ("down", n, inner)):
        a[m] = (on(at(m + "_packed"), count, rows, cols // 2, dtype=U8), on(at(m + "_codes"), count, rows, cols // 16, dtype=U8),
                on(at(m + "_scale"), count, dtype=F32))
    return a


MATRICES = [f"{m}_{part}" for m in ("gate", "up", "down") for part in ("packed", "codes", "scale")]


@pytest.mark.parametrize("name", ["x", "y", "ids", "weights", "ws", "all"] + MATRICES)
def test_experts(name):
    a = layer(**{name: 1})
    with pytest.raises(ValueError):
        hs.hscale_experts(a["x"], a["ids"], a["weights"], a["gate"], a["up"], a["down"], 0, a["y"], a["ws"])


@pytest.mark.parametrize("name", ["dy", "x", "y", "ids", "weights", "dweights", "ws", "all"] + MATRICES)
def test_experts_backward(name):
    a = layer(**{name: 1})
    with pytest.raises(ValueError):
        hs.hscale_experts_backward(a["dy"], a["x"], a["ids"], a["weights"], a["gate"], a["up"], a["down"], 0, a["y"], a["dweights"],
                                   a["ws"])


@pytest.mark.parametrize("name", ["logits", "ids", "weights", "dweights", "dlogits", "all"])
def test_router(name):
    at = lambda n: 1 if name in (n, "all") else 0  # noqa: E731
    logits, dlogits = on(at("logits"), 3, 8, dtype=F32), on(at("dlogits"), 3, 8, dtype=F32)
    ids, weights = on(at("ids"), 3, 2, dtype=I32), on(at("weights"), 3, 2, dtype=F32)
    dweights = on(at("dweights"), 3, 2, dtype=F32)
    if name not in ("dweights", "dlogits"):
        with pytest.raises(ValueError):
            hs.hscale_route(logits, ids, weights, True)
    with pytest.raises(ValueError):
        hs.hscale_route_backward(logits, ids, weights, dweights, False, dlogits)


@pytest.mark.parametrize("name", ["tensors", "norm", "out", "ws", "all"])
def test_clip(name):
    at = lambda n: 1 if name in (n, "all") else 0  # noqa: E731
    grads, out = [on(at("tensors"), 8, dtype=F32)], [on(at("out"), 8, dtype=F32)]
    norm, ws = on(at("norm"), 1, dtype=F32), on(at("ws"), 8192, dtype=U8)
    if name != "out":
        with pytest.raises(ValueError):
            hs.hscale_grad_norm(grads, norm, ws)
    with pytest.raises(ValueError):
        hs.hscale_grad_clip(grads, 1.0, norm, out, ws)
    with pytest.raises(ValueError):
        hs.hscale_tensors([on(0, 8, dtype=F32), on(1, 8, dtype=F32)])
