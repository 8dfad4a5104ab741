"""Host bounds of a paged batch that are left out."""
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


@pytest.mark.parametrize("new", [1, 40])
def test_bounds_that_are_left_out_are_those_of_the_table(new):
    """Without max_q_len and max_seq_len the call is planned for what the table and q can hold: the same bits as with
    those bounds given."""
    bt = R.Batch([1024, 700], [new] * 2, 8, 8, 128, 64, seed=6, max_pages=16)
    a = attend(bt, max_q=2 * new, max_seq=1024)
    cache, batch = bt.handles(P)
    default = P.PagedBatch(batch.page_table, batch.seq_lens, batch.q_starts, bt.T)
    out, lse = torch.empty_like(a[0]), torch.empty_like(a[1])
    ws = torch.empty(P.sasq_paged_attention_workspace(cache, default, 8), dtype=torch.uint8, device="cuda")
    P.sasq_paged_attention(cache, default, bt.q, out, ws, lse=lse)
    assert torch.equal(out.view(torch.int16), a[0].view(torch.int16)) and torch.equal(lse, a[1])
