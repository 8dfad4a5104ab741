"""What the 4-bit linear's entry points refuse on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

import paper_2512_14481_b200 as P

OK, INVALID, UNSUPPORTED = 0, 1, 2


@pytest.fixture(scope="module")
def addr():
    buf = (ctypes.c_char * 512)()
    yield (ctypes.addressof(buf) + 63) & ~63          # never dereferenced: every call must fail, or have nothing to do


def linear(a, **kw):
    d = dict(x=a, w=a, s=a, bias=None, y=a + 64, T=3, N=8, K=256, group=128, dt=1)
    d.update(kw)
    return P.load_library().sasq_w4_linear(d["x"], d["w"], d["s"], d["bias"], d["y"], d["T"], d["N"], d["K"], d["group"], d["dt"], None)


def quantize(a, **kw):
    d = dict(w=a, c=a, s=a, N=8, K=256, group=128, dt=1)
    d.update(kw)
    return P.load_library().sasq_quantize_weight_w4(d["w"], d["c"], d["s"], d["N"], d["K"], d["group"], d["dt"], None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(s=None), INVALID), (dict(y=None), INVALID), (dict(T=-1), INVALID),
    (dict(N=0), INVALID), (dict(N=-1), INVALID), (dict(K=0), INVALID), (dict(K=-128), INVALID), (dict(dt=2), INVALID),
    (dict(group=16), UNSUPPORTED), (dict(group=256), UNSUPPORTED), (dict(group=0), UNSUPPORTED), (dict(group=-32), UNSUPPORTED),
    (dict(K=192), UNSUPPORTED), (dict(K=1 << 25), UNSUPPORTED), (dict(N=1 << 31), UNSUPPORTED), (dict(T=1 << 21), UNSUPPORTED),
    (dict(T=0, x=None, y=None), OK)])
def test_linear(addr, change, status):
    assert linear(addr, **change) == status


def test_alignment_and_aliases(addr):
    for name in ("x", "w", "s", "bias", "y"):
        assert linear(addr, **{name: addr + 8}) == INVALID
    assert linear(addr, y=addr) == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(w=None), INVALID), (dict(c=None), INVALID), (dict(s=None), INVALID), (dict(N=-1), INVALID), (dict(K=0), INVALID),
    (dict(dt=-1), INVALID), (dict(group=48), UNSUPPORTED), (dict(K=160), UNSUPPORTED), (dict(w=1), INVALID), (dict(N=0, w=None), OK)])
def test_quantizer(addr, change, status):
    assert quantize(addr, **change) == status


def test_binding_refuses_cpu_tensors():
    import torch
    x, w, s = torch.zeros((1, 64)).half(), torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((8, 2)).half()
    with pytest.raises(TypeError):
        P.sasq_w4_linear(x, w, s, torch.zeros((1, 8)).half())
    with pytest.raises(TypeError):
        P.sasq_quantize_weight_w4(torch.zeros((8, 64)), w, s)


def test_the_most_tokens_and_columns(addr):
    assert linear(addr, T=(1 << 19) + 1) == UNSUPPORTED and linear(addr, K=(1 << 24) + 128) == UNSUPPORTED
    assert linear(addr, N=(1 << 30) + 1) == UNSUPPORTED
