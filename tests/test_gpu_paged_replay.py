"""Replays of a captured attention call from a graph, up to the bounds that it was captured with."""
import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("new", [1, 3, 60])
def test_replays_up_to_the_captured_bounds(new, int8):
    """One captured call, replayed on other lengths, pages and values: up to the bound of the keys and all of the table's
    entries, a sequence without context, one without keys; out and lse are compared after each."""
    most, page = 1280, 32
    bt = R.Batch([most, most], [new] * 2, 8, 4, 128, page, int8=int8, seed=1, max_pages=most // page)
    cache, batch = bt.handles(P, max_seq=most)
    out = torch.empty((bt.T, 8, 128), dtype=bt.dtype, device="cuda")
    lse = torch.empty((bt.T, 8), device="cuda")
    ws = torch.empty(P.sasq_paged_attention_workspace(cache, batch, 8), dtype=torch.uint8, device="cuda")
    P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse)
    for seed, lens in ((11, [64, 1100]), (12, [most, new]), (13, [0, most - 1]), (14, [most, most])):
        other = R.Batch(lens, [new] * 2, 8, 4, 128, page, int8=int8, seed=seed, max_pages=most // page)
        n = other.k.shape[0]
        assert n <= bt.k.shape[0]
        bt.k[:n].copy_(other.k)
        bt.v[:n].copy_(other.v)
        if int8:
            cache.k_scale.copy_(other.k_scale)
            cache.v_scale.copy_(other.v_scale)
        bt.q.copy_(other.q)
        batch.page_table.copy_(torch.from_numpy(other.table))
        batch.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(7.0)
        lse.fill_(7.0)
        ws.fill_(255)
        graph.replay()
        assert P.sasq_device_status() == 0
        want, want_lse, tol, lse_tol = R.attention(other, 128 ** -0.5, True)
        assert (np.abs(out.float().cpu().double().numpy() - want) <= tol).all()
        got = lse.cpu().double().numpy()
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got), empty)
        assert (np.abs(got[~empty] - want_lse[~empty]) <= lse_tol[~empty]).all()
