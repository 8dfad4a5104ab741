"""The paged operators' binding takes tensors of one device, the current one (no GPU needed: the tensors say where they are).
No call here reaches a launch: it is refused, or has no tokens."""
import pytest
import torch

import paper_2512_14481_b200 as P
from paper_2512_14481_b200 import binding


class Says(torch.Tensor):
    """A host tensor that claims to lie on CUDA device `index`."""
    index = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.index


class SaysOne(Says):
    index = 1


def on(device, t):
    return t.as_subclass(SaysOne if device else Says)


def handles(cache=0, batch=0, tokens=0, **other):
    at = lambda name, where: other.get(name, where)  # noqa: E731
    pool = lambda w: on(w, torch.zeros((3, 16, 2, 64), dtype=torch.int8))  # noqa: E731
    i32 = lambda w, *n: on(w, torch.zeros(n, dtype=torch.int32))  # noqa: E731
    c = P.KVCache(pool(cache), pool(at("v_pool", cache)), on(at("k_scale", cache), torch.ones(2)), on(at("v_scale", cache), torch.ones(2)))
    return c, P.PagedBatch(i32(batch, 1, 3), i32(at("lens", batch), 1), i32(at("starts", batch), 2), tokens)


def rows(w, heads):
    return on(w, torch.zeros((0, heads, 64), dtype=torch.bfloat16))


@pytest.fixture(autouse=True)
def first_device_is_current(monkeypatch):
    monkeypatch.setattr(binding, "_current_device", lambda: 0, raising=False)


@pytest.mark.parametrize("which", ["v_pool", "k_scale", "v_scale", "lens", "starts"])
def test_handles_of_two_devices(which):
    handles()
    with pytest.raises(ValueError):
        handles(**{which: 1})


def append(c, b, **w):
    at = lambda name: w.get(name, 0)  # noqa: E731
    P.sasq_rope_kv_append(c, b, rows(at("q"), 4), rows(at("k"), 2), rows(at("v"), 2), rows(at("q_out"), 4),
                          on(at("cos_sin"), torch.zeros((8, 64))), stream=0)


def attend(c, b, **w):
    at = lambda name: w.get(name, 0)  # noqa: E731
    P.sasq_paged_attention(c, b, rows(at("q"), 4), rows(at("out"), 4), on(at("ws"), torch.zeros(16, dtype=torch.uint8)),
                           lse=on(at("lse"), torch.zeros((0, 4))), stream=0)


@pytest.mark.parametrize("call,names", [(append, ("q", "k", "v", "q_out", "cos_sin")), (attend, ("q", "out", "ws", "lse"))])
def test_calls_with_tensors_of_two_devices(call, names):
    call(*handles())                                          # no tokens: nothing to launch, and nothing to refuse
    for name in names:
        with pytest.raises(ValueError):
            call(*handles(), **{name: 1})
    with pytest.raises(ValueError):
        call(*handles(cache=1, batch=0))
    with pytest.raises(ValueError):
        call(*handles(cache=0, batch=1))


@pytest.mark.parametrize("call,names", [(append, ("q", "k", "v", "q_out", "cos_sin")), (attend, ("q", "out", "ws", "lse"))])
def test_calls_on_a_device_that_is_not_current(call, names, monkeypatch):
    everything = {name: 1 for name in names}
    with pytest.raises(ValueError):
        call(*handles(cache=1, batch=1), **everything)
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    call(*handles(cache=1, batch=1), **everything)
