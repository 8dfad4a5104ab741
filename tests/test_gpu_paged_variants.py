"""Every kernel variant of the paged attention that a rule on sizes can choose, on sizes that reach it: one and two blocks
of eight rows; an item to a cluster of four- and of eight-warp blocks, equal stretches with the joining launch, and the
many-row kernel beside them; both types, both caches, both head dimensions."""
import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu


def attend(bt, max_q=None, max_seq=None):
    cache, batch = bt.handles(P, max_q, max_seq)
    out = torch.full((bt.T, bt.heads, bt.dim), 7.0, dtype=bt.dtype, device="cuda")
    lse = torch.full((bt.T, bt.heads), 7.0, device="cuda")
    ws = torch.full((max(16, P.sasq_paged_attention_workspace(cache, batch, bt.heads)),), 255, dtype=torch.uint8, device="cuda")
    P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse)
    assert P.sasq_device_status() == 0
    return out, lse


def check(bt):
    out, lse = attend(bt)
    want, want_lse, tol, lse_tol = R.attention(bt, bt.dim ** -0.5, True)
    assert (np.abs(out.float().cpu().double().numpy() - want) <= tol).all()
    got = lse.cpu().double().numpy()
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(got), empty)
    assert (np.abs(got[~empty] - want_lse[~empty]) <= lse_tol[~empty]).all()


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,count,hi", [
    (1, 3, 900),        # 4 rows, few items: clusters of eight-warp blocks
    (1, 14, 900),       # 4 rows, 28 items: clusters of four-warp blocks
    (2, 60, 400),       # 8 rows, many items: equal stretches
    (1, 2, 14000),      # 4 rows, long keys: equal stretches
    (3, 2, 900),        # 12 rows, clusters
    (4, 14, 600),       # 16 rows, clusters of four-warp blocks
    (3, 60, 400),       # 12 rows, equal stretches
    (4, 3, 14000),      # 16 rows, long keys: equal stretches
    (5, 3, 900),        # 20 rows: two row tiles, clusters
    (16, 2, 700),       # 64 rows: four row tiles, clusters
    (17, 2, 700),       # 68 rows: the many-row kernel
    (9, 30, 300)])      # 36 rows of many sequences: the many-row kernel
def test_rows_and_items(new, count, hi, dim, dtype, int8):
    lens = [max(0, hi - (hi * i) // count - (3 * i) % 5) for i in range(count)]
    check(R.Batch(lens, [max(1, new - i % 2) if i else new for i in range(count)], 8, 2, dim, 32, dtype, int8, seed=new + count))


def test_one_head_or_one_page_needs_no_stride():
    """The C entries with a stride of zero for a dimension of one entry."""
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    for pages, K in ((3, 1), (1, 2)):
        k, v = (torch.randn((pages, 16, K, 64), device="cuda").to(torch.bfloat16) for _ in range(2))
        q = torch.randn((144, 2 * K, 64), device="cuda").to(torch.bfloat16)
        batch = P.PagedBatch(i32([[0]]), i32([16]), i32([0, 144]), 144, 144, 16)
        outs = []
        for zero in (False, True):
            cache = P.KVCache(k, v)
            if zero:
                name = "head_stride" if K == 1 else "page_stride"
                setattr(cache.struct, name, 0)
            out = torch.empty_like(q)
            ws = torch.empty(P.sasq_paged_attention_workspace(cache, batch, 2 * K), dtype=torch.uint8, device="cuda")
            P.sasq_paged_attention(cache, batch, q, out, ws)
            outs.append(out)
        assert P.sasq_device_status() == 0 and torch.equal(outs[0], outs[1])
