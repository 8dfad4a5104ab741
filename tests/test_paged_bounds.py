"""Host bounds of a paged batch beyond what q and the page table can hold plan nothing else than those (no GPU needed)."""
import ctypes

import pytest

import paper_2512_14481_b200 as P


def workspace(kv_heads, dim, kind, group, **bounds):
    address = 4096                                   # never dereferenced
    scale = address if kind == P.SASQ_KV_INT8 else None
    cache = P.KVCacheStruct(address, address, scale, scale, 16 * kv_heads * dim, kv_heads * dim, dim, 100, 16, kv_heads, dim, kind)
    batch = P.KVBatchStruct(address, address, address, 8, 3, 8, bounds.pop("total_q"), bounds.pop("max_q_len"), bounds.pop("max_seq_len"), 0)
    return P.load_library().sasq_paged_attention_workspace(ctypes.byref(cache), ctypes.byref(batch), kv_heads * group)


@pytest.mark.parametrize("kind", [P.SASQ_KV_16BIT, P.SASQ_KV_INT8])
@pytest.mark.parametrize("kv_heads,dim,group", [(1, 64, 1), (2, 128, 4), (1, 128, 130)])
@pytest.mark.parametrize("total_q", [1, 3, 40])
def test_workspace_of_wide_open_bounds(total_q, kv_heads, dim, group, kind):
    room = 8 * 16
    given = workspace(kv_heads, dim, kind, group, total_q=total_q, max_q_len=total_q, max_seq_len=room)
    assert given > 0
    for q, s in ((0x7FFFFFFF, room), (total_q, 0x7FFFFFFF), (total_q + 1, room + 1)):
        assert workspace(kv_heads, dim, kind, group, total_q=total_q, max_q_len=q, max_seq_len=s) == given
