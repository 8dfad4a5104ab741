"""Append to a 4-bit cache: rows that no sequence owns, before the first and behind the last, have no part in anything."""
import numpy as np
import pytest
import torch

import kv4_reference as R4
import paper_2512_14481_b200 as P
from test_gpu_paged_append import table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 3, 400])
@pytest.mark.parametrize("fill", [0.0, float("nan"), float("inf")])
def test_padding_on_both_sides(new, fill):
    lead, tail = 5, 300
    lens = [new + 7, new, 500]
    bt = R4.Batch(lens, [new] * 3, 6, 2, 64, 32, torch.bfloat16, seed=new)
    g = torch.Generator().manual_seed(2)
    qkv = torch.randn((bt.T, 10, 64), generator=g).to(torch.bfloat16)
    cs = torch.from_numpy(table(520, 64)).cuda()
    stored = []
    for before, behind in ((0, 0), (lead, tail)):
        cache, batch = bt.handles(P)
        k0, v0 = cache.k.clone(), cache.v.clone()
        wide = torch.full((before + bt.T + behind, 10, 64), fill, dtype=torch.bfloat16, device="cuda")
        wide[before:before + bt.T] = qkv.cuda()
        starts = torch.from_numpy(bt.starts.astype(np.int32) + before).cuda()
        padded = P.PagedBatch(batch.page_table, batch.seq_lens, starts, wide.shape[0], new, 507)
        q_out = torch.full((wide.shape[0], 6, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        P.sasq_rope_kv_append(cache, padded, wide[:, :6], wide[:, 6:8], wide[:, 8:], q_out, cs)
        assert P.sasq_device_status() == 0
        assert (q_out[:before] == 7.0).all() and (q_out[before + bt.T:] == 7.0).all()
        stored.append((cache.k.clone(), cache.v.clone(), q_out[before:before + bt.T]))
        assert not torch.equal(cache.k, k0)
        cache.k.copy_(k0), cache.v.copy_(v0)
    for a, b in zip(*stored):
        assert torch.equal(a, b)
