"""Attention over a 4-bit cache against a plain one in 64 bits."""
import numpy as np
import pytest
import torch

import kv4_reference as R4
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu


def attend(bt, causal=True, scale=None, max_q=None, max_seq=None):
    cache, batch = bt.handles(P, max_q, max_seq)
    out = torch.full((bt.T, bt.heads, bt.dim), 7.0, dtype=bt.dtype, device="cuda")
    lse = torch.full((bt.T, bt.heads), 7.0, device="cuda")
    ws = torch.full((max(16, P.sasq_paged_attention_workspace(cache, batch, bt.heads)),), 255, dtype=torch.uint8, device="cuda")
    P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse, scale=scale, causal=causal)
    assert P.sasq_device_status() == 0
    return out, lse


def check(bt, causal=True, scale=None, **kw):
    out, lse = attend(bt, causal, scale, **kw)
    want, want_lse, tol, lse_tol = R4.attention(bt, bt.dim ** -0.5 if scale is None else scale, causal)
    got, got_lse = out.float().cpu().double().numpy(), lse.cpu().double().numpy()
    own = ~np.isnan(want)
    assert (np.abs(got - want)[own] <= tol[own]).all()
    assert (got[~own] == 7.0).all()                        # rows behind the last sequence
    rows = ~np.isnan(want_lse)
    empty = np.isneginf(want_lse)
    assert (got_lse[~rows] == 7.0).all() and np.array_equal(np.isneginf(got_lse), empty)
    seen = rows & ~empty
    assert (np.abs(got_lse[seen] - want_lse[seen]) <= lse_tol[seen]).all()
    return out, lse


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
    (17, 2, 700),       # 68 rows
    (9, 30, 300)])      # 36 rows of many sequences
def test_rows_and_items(new, count, hi, dim, dtype):
    lens = [max(0, hi - (hi * i) // count - (3 * i) % 5) for i in range(count)]
    check(R4.Batch(lens, [max(1, new - i % 2) if i else new for i in range(count)], 8, 2, dim, 32, dtype, seed=new + count))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 1), (10, 2), (7, 1), (24, 2), (12, 12), (130, 1)])
def test_groups(heads, kv_heads, causal):
    check(R4.Batch([70, 1, 0, 300], [3, 1, 2, 40], heads, kv_heads, 64, 16, torch.float16, seed=heads), causal)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("tokens_first", [False, True])
@pytest.mark.parametrize("new", [1, 100])
def test_pages_and_orders(page, tokens_first, new):
    check(R4.Batch([new, page + new, 3 * page + 1 + new, 1], [new, new, new, 1], 4, 2, 128, page, torch.bfloat16, tokens_first, seed=page))


@pytest.mark.parametrize("new", [1, 2, 40, 300])
def test_lengths_around_units(new):
    """Keys up to, at and past the ends of the kernels' steps, units and tiles."""
    lens = [new + k for k in (0, 1, 14, 15, 16, 17, 31, 32, 63, 64, 65, 127, 128, 129, 255, 256, 257)]
    check(R4.Batch(lens, [new] * len(lens), 4, 2, 64, 16, torch.float16, seed=new))


@pytest.mark.parametrize("causal", [True, False])
def test_rows_without_keys_padding_and_queries_apart(causal):
    bt = R4.Batch([2, 0, 9, 130], [6, 3, 0, 130], 4, 2, 128, 16, torch.bfloat16, seed=5, pad_rows=5, q_extra=3)
    out, lse = check(bt, causal)
    if causal:
        assert (out[:4] == 0).all() and torch.isneginf(lse[:4]).all()
    assert (out[6:9] == 0).all() and torch.isneginf(lse[6:9]).all()


@pytest.mark.parametrize("new", [1, 30])
@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0, 1e-30])
def test_scales(scale, new):
    check(R4.Batch([200, 33], [new, new], 4, 2, 64, 16, torch.bfloat16, seed=8), scale=scale)


@pytest.mark.parametrize("new", [1, 5, 50])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_few_channels_show_every_bit(dtype, new):
    """One or two non-zero elements a query row: nothing but the operands' own rounding could be off, and it must not be."""
    bt = R4.Batch([150, 90], [new, new], 4, 2, 128, 16, dtype, seed=3)
    keep = torch.zeros_like(bt.q_wide)
    t = torch.arange(bt.T)[:, None]
    h = torch.arange(4)[None]
    keep[t, h, (17 * t + 5 * h) % 128] = 1
    keep[t, h, (31 * t + 3 * h) % 128] = 1
    bt.q_wide = bt.q_wide * keep
    bt.q = bt.q_wide.cuda()
    check(bt)


@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("q_by,f_by", [(2.0 ** 30, 2.0 ** -30), (2.0 ** -40, 2.0 ** 40), (2.0 ** 90, 2.0 ** -90), (1.0, -1.0)])
def test_far_queries_and_factors(new, q_by, f_by):
    bt = R4.Batch([150, 90], [new, new], 4, 2, 64, 16, torch.bfloat16, seed=4)
    bt.q_wide = bt.q_wide * q_by
    bt.q = bt.q_wide.cuda()
    bt.k_scale, bt.v_scale = bt.k_scale * f_by, -bt.v_scale
    check(bt)


@pytest.mark.parametrize("new", [1, 50])
def test_a_nan_in_a_query_stays_in_its_row(new):
    bt = R4.Batch([150, 90], [new, new], 4, 2, 64, 16, torch.bfloat16, seed=4)
    want, want_lse = attend(bt)
    bt.q_wide[0, 1, 5] = float("nan")
    bt.q = bt.q_wide.cuda()
    out, lse = attend(bt)
    assert torch.isnan(out[0, 1]).all() and torch.isnan(lse[0, 1])
    out[0, 1], lse[0, 1] = want[0, 1], want_lse[0, 1]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("new", [1, 50])
def test_loud_and_faint_keys(new):
    """One key far above many others, at the end and at the beginning."""
    for at in (0, 699):
        bt = R4.Batch([700], [new], 2, 1, 64, 16, torch.float16, seed=6)
        bt.k_scale = torch.full((1, 64), 0.25)
        k = bt.k_host.clone() // 4
        q = torch.full((bt.T, 2, 64), 1.0).to(torch.float16)
        k[int(bt.table[0, at // 16]), at % 16] = 7
        bt.set_codes(k, bt.v_host)
        bt.q_wide, bt.q = q, q.cuda()
        check(bt, causal=False)


@pytest.mark.parametrize("new", [1, 50])
def test_bad_pages_and_factors_are_reported(new):
    bt = R4.Batch([100, 100], [new, new], 2, 2, 64, 16, seed=1)
    good = bt.table[0, 2]
    cache, batch = bt.handles(P)
    out = torch.zeros((bt.T, 2, 64), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(16, P.sasq_paged_attention_workspace(cache, batch, 2)), dtype=torch.uint8, device="cuda")
    for wrong in (-1, 1 << 20):
        bt.table[0, 2] = wrong
        cache, batch = bt.handles(P)
        P.sasq_paged_attention(cache, batch, bt.q, out, ws)
        assert P.sasq_device_status() == 7
    bt.table[0, 2] = good
    for name in ("k_scale", "v_scale"):
        for bad in (0.0, float("nan"), 3.4e38):
            cache, batch = bt.handles(P)
            getattr(cache, name)[1, 37] = bad
            P.sasq_paged_attention(cache, batch, bt.q, out, ws)
            assert P.sasq_device_status() == 4


@pytest.mark.parametrize("new", [1, 50])
def test_replayed_and_from_run_to_run(new):
    bt = R4.Batch([700, 90, 33], [new, new, 3], 8, 2, 128, 32, torch.bfloat16, seed=9)
    cache, batch = bt.handles(P, max_seq=700)
    out, lse = torch.empty((bt.T, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((bt.T, 8), device="cuda")
    ws = torch.empty(max(16, P.sasq_paged_attention_workspace(cache, batch, 8)), dtype=torch.uint8, device="cuda")
    call = lambda: P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse)  # noqa: E731
    call()
    first, first_lse = out.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    out.zero_(), lse.zero_()
    graph.replay()
    assert torch.equal(out, first) and torch.equal(lse, first_lse)
    bt.seq_lens = [640, 50, 3]
    batch.seq_lens.copy_(torch.tensor(bt.seq_lens, dtype=torch.int32))
    graph.replay()
    want, _, tol, _ = R4.attention(bt, 128 ** -0.5, True)
    assert (np.abs(out.float().cpu().double().numpy() - want) <= tol).all()
