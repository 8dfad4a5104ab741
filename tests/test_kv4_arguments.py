"""What the paged entry points refuse of a 4-bit cache on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

import paper_2512_14481_b200 as P
from test_paged_arguments import INVALID, OK, UNSUPPORTED, WORKSPACE, addr, append, attend, batch, cache  # noqa: F401


def cache4(a, **kw):
    return cache(a, **{**dict(kind=P.SASQ_KV_INT4, k_scale=a, v_scale=a), **kw})


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("change,status", [
    (dict(k=None), INVALID), (dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID), (dict(kind=3), INVALID),
    (dict(kind=-1), INVALID), (dict(head_stride=64 + 16), INVALID), (dict(token_stride=4 * 64 + 16), INVALID),
    (dict(page_stride=16 * 4 * 64 + 8), INVALID), (dict(page_size=48), UNSUPPORTED)])
def test_caches(addr, call, change, status):  # noqa: F811
    assert call(cache4(addr, **change), batch(addr), addr) == status


@pytest.mark.parametrize("call", [append, attend])
def test_factors_are_read_in_words(addr, call):  # noqa: F811
    assert call(cache4(addr, k_scale=addr + 4), batch(addr), addr) == INVALID
    assert call(cache4(addr, v_scale=addr + 8), batch(addr), addr) == INVALID
    assert call(cache4(addr), batch(addr, total_q=0), addr) == OK


@pytest.mark.parametrize("dim", [16, 48, 80, 240, 288])
def test_append_head_dims(addr, dim):  # noqa: F811
    wide = -(-dim // 32) * 32
    c = cache4(addr, head_dim=dim, head_stride=wide, token_stride=4 * wide, page_stride=64 * wide)
    assert append(c, batch(addr), addr, qs=8 * dim, ks=4 * dim, vs=4 * dim, qos=8 * dim, rot=0) == UNSUPPORTED


def test_attention_head_dims_and_workspace(addr):  # noqa: F811
    for dim in (32, 96, 256):
        c = cache4(addr, head_dim=dim, head_stride=dim, token_stride=4 * dim, page_stride=64 * dim)
        assert attend(c, batch(addr), addr, qs=8 * dim, os=8 * dim) == UNSUPPORTED
    assert attend(cache4(addr), batch(addr), addr, ws=None) == WORKSPACE
    assert attend(cache4(addr), batch(addr), addr, nbytes=64) == WORKSPACE
    assert P.load_library().sasq_paged_attention_workspace(ctypes.byref(cache4(addr)), ctypes.byref(batch(addr)), 8) > 0
