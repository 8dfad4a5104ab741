"""Attention over the paged cache against a 64-bit reference, at the sizes, masks and layouts where it can go wrong.
Tolerances are derived in paged_reference.attention."""
import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu


def attend(bt, scale=None, causal=True, max_q=None, max_seq=None, with_lse=True, stream=None):
    cache, batch = bt.handles(P, max_q, max_seq)
    out = torch.full((bt.T, bt.heads, bt.dim), 7.0, dtype=bt.dtype, device="cuda")
    lse = torch.full((bt.T, bt.heads), 7.0, device="cuda") if with_lse else None
    ws = torch.full((max(16, P.sasq_paged_attention_workspace(cache, batch, bt.heads)),), 255, dtype=torch.uint8, device="cuda")
    P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse, scale=scale, causal=causal, stream=stream)
    return out, lse


def check(bt, scale=None, causal=True, **kw):
    out, lse = attend(bt, scale, causal, **kw)
    assert P.sasq_device_status() == 0
    want, want_lse, tol, lse_tol = R.attention(bt, bt.dim ** -0.5 if scale is None else scale, causal)
    got, got_lse = out.float().cpu().double().numpy(), lse.cpu().double().numpy()
    own = slice(0, int(bt.starts[-1]))
    bad = ~(np.abs(got[own] - want[own]) <= tol[own])
    assert not bad.any(), f"{bad.sum()} of {bad.size} outputs off, first at {np.argwhere(bad)[0]}: " \
        f"{got[own][bad][0]} for {want[own][bad][0]} +- {tol[own][bad][0]}"
    empty = ~np.isfinite(want_lse[own])
    assert np.array_equal(np.isneginf(got_lse[own]), empty)
    assert (got[own][empty] == 0).all()
    fine = ~empty
    assert (np.abs(got_lse[own][fine] - want_lse[own][fine]) <= lse_tol[own][fine]).all()
    assert (got[own.stop:] == 7).all() and (got_lse[own.stop:] == 7).all()      # padding rows stay as they were


SHAPES = [  # heads, kv_heads, dim
    (4, 4, 128), (8, 2, 128), (10, 2, 64), (7, 1, 128), (16, 1, 64), (6, 2, 128)]


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
def test_single_tokens(heads, kv_heads, dim, dtype, int8):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 400, 1000]
    check(R.Batch(lens, [1] * len(lens), heads, kv_heads, dim, 16, dtype, int8, seed=heads))


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
def test_ragged_chunks(heads, kv_heads, dim, dtype, int8):
    new = [1, 3, 16, 33, 100, 129, 300, 0, 257]
    lens = [1, 70, 16, 500, 101, 400, 300, 50, 640]
    check(R.Batch(lens, new, heads, kv_heads, dim, 32, dtype, int8, seed=dim + heads, q_extra=2))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("tokens_first", [True, False])
@pytest.mark.parametrize("new", [2, 90])
def test_pages_and_orders(page, tokens_first, causal, new):
    lens = [new, page - 1 + new, page + new, 2 * page + 1 + new, 777]
    for int8 in (False, True):
        check(R.Batch(lens, [new] * 5, 8, 4, 128, page, torch.bfloat16, int8, tokens_first, seed=page), causal=causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new", [1, 5, 200])
def test_rows_without_keys(new, causal):
    """Sequences shorter than their chunk (the first tokens have no place), and empty ones."""
    lens = [0, new, max(0, new - 1), new // 2, new + 40, 0]
    for int8 in (False, True):
        check(R.Batch(lens, [new] * 6, 8, 2, 64, 16, torch.float16, int8, seed=new), causal=causal)


@pytest.mark.parametrize("new", [1, 40])
def test_bounds_of_the_host_are_hints(new):
    """Too small an upper bound costs time and not results; too large a one neither."""
    bt = R.Batch([300, 40 + new, 1000], [new] * 3, 8, 4, 128, 16, seed=3)
    check(bt, max_q=1, max_seq=1)
    check(bt, max_q=5000, max_seq=1 << 20)


def test_padding_rows_and_empty_batches():
    check(R.Batch([40, 90], [3, 50], 4, 2, 128, 16, pad_rows=30))
    check(R.Batch([40, 90], [0, 0], 4, 2, 128, 16, pad_rows=4))
    check(R.Batch([40, 90], [0, 0], 4, 2, 128, 16))


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
@pytest.mark.parametrize("new", [1, 70])
def test_scales(scale, new):
    check(R.Batch([new, 500], [new] * 2, 4, 4, 64, 64, seed=5), scale=scale)


@pytest.mark.parametrize("new", [1, 150])
def test_logits_that_grow_and_fall(new):
    """Keys sorted by loudness, rising and falling: the running maximum moves at every step, or never again."""
    for flip in (False, True):
        bt = R.Batch([1500], [new], 4, 2, 128, 64, torch.float16, seed=9, tokens_first=True)
        loud = torch.linspace(0.01, 3.0, 1500)
        loud = loud.flip(0) if flip else loud
        pos = np.arange(1500)
        page, row = torch.from_numpy(bt.table[0, pos // 64].astype(np.int64)), torch.from_numpy(pos % 64)
        bt.k_host[page, row] = (bt.k_host[page, row].float() * loud[:, None, None]).to(bt.dtype)
        bt.k.copy_(bt.k_host)
        check(bt)


@pytest.mark.parametrize("new", [1, 64])
def test_every_run_has_the_same_bits(new):
    bt = R.Batch([3000, 100, 1777], [new] * 3, 16, 4, 128, 16, seed=2)
    first, first_lse = attend(bt)
    for _ in range(3):
        out, lse = attend(bt)
        assert torch.equal(out.view(torch.int16), first.view(torch.int16)) and torch.equal(lse, first_lse)
    out, _ = attend(bt, with_lse=False)
    assert torch.equal(out.view(torch.int16), first.view(torch.int16))


def test_many_sequences():
    """More sequences than a block has threads."""
    lens = [(37 * i) % 90 for i in range(1500)]
    check(R.Batch(lens, [1 if i % 7 else 0 for i in range(1500)], 2, 1, 64, 16, seed=4))


def test_offsets_beyond_32_bits():
    """Pages further than 2^31 elements into the pool."""
    pages, page, K, D = 140000, 128, 1, 128                       # 4.6 GB per tensor
    k = torch.zeros((pages, page, K, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    bt = R.Batch([700, 300], [1, 200], 4, K, D, page, seed=6)
    n = bt.k_host.shape[0]
    k[-n:], v[-n:] = bt.k, bt.v
    bt.k, bt.v = k, v
    host = bt.table.copy()
    bt.table = np.where(host >= 0, host + pages - n, -1).astype(np.int32)
    out, lse = attend(bt)
    assert P.sasq_device_status() == 0
    bt.table = host
    want, _, tol, _ = R.attention(bt, D ** -0.5, True)
    assert (np.abs(out.float().cpu().double().numpy() - want) <= tol).all()


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim,new,lens", [
    (32, 32, 128, [300, 40, 257], [1500, 900, 2300]),       # several units and items per block, both row tiles in use
    (24, 24, 128, [20, 33, 7], [3000, 2000, 1111]),         # rows for one row tile, long keys
    (40, 8, 64, [7, 90, 33], [4000, 3000, 1800]),
    (8, 8, 64, [1000, 129], [1700, 1900]),
    (64, 64, 128, [1, 1, 1, 1], [700, 40, 3000, 1]),        # more units than blocks, single tokens
])
def test_more_work_than_blocks(heads, kv_heads, dim, new, lens, int8):
    check(R.Batch(lens, new, heads, kv_heads, dim, 64, torch.float16 if dim == 64 else torch.bfloat16, int8, seed=heads + dim))


@pytest.mark.parametrize("new", [1, 60])
def test_other_stream_and_graph(new):
    """On a stream of its own, and replayed from a graph on new values, lengths and pages."""
    bt = R.Batch([900, 333], [new] * 2, 8, 8, 128, 32, seed=1, max_pages=40)
    cache, batch = bt.handles(P, max_seq=1280)
    out = torch.empty((bt.T, 8, 128), dtype=bt.dtype, device="cuda")
    lse = torch.empty((bt.T, 8), device="cuda")
    ws = torch.empty(P.sasq_paged_attention_workspace(cache, batch, 8), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse)
    side.synchronize()
    want, _, tol, _ = R.attention(bt, 128 ** -0.5, True)
    assert (np.abs(out.float().cpu().double().numpy() - want) <= tol).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse)
    for seed, lens in ((11, [64, 1100]), (12, [1280, new])):
        other = R.Batch(lens, [new] * 2, 8, 8, 128, 32, seed=seed, max_pages=40)
        pool = bt.k.shape[0]
        if other.k.shape[0] > pool:
            continue
        bt.k[:other.k.shape[0]].copy_(other.k)
        bt.v[:other.k.shape[0]].copy_(other.v)
        bt.q.copy_(other.q)
        batch.page_table.copy_(torch.from_numpy(other.table))
        batch.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        want, _, tol, _ = R.attention(other, 128 ** -0.5, True)
        assert (np.abs(out.float().cpu().double().numpy() - want) <= tol).all()
    assert P.sasq_device_status() == 0


def test_pages_outside_the_cache_are_reported():
    """The access is skipped, the status word says so, and the other sequence is right."""
    for new in (1, 50):
        bt = R.Batch([200, 200], [new] * 2, 4, 4, 128, 16, seed=8)
        good = bt.table[0, 3]
        for wrong in (-1, 1 << 20):
            bt.table[0, 3] = wrong
            out, _ = attend(bt)
            assert P.sasq_device_status() == 7
            bt.table[0, 3] = good
            want, _, tol, _ = R.attention(bt, 128 ** -0.5, True)
            assert (np.abs(out.float().cpu().double().numpy() - want) <= tol)[new:].all()
        bt.seq_lens[0] = 5000                                        # more keys than its table has room for
        attend(bt)
        assert P.sasq_device_status() == 7


@pytest.mark.parametrize("int8", [False, True])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_clean(int8):
    """The many-row kernel with a wait limit of zero cycles: it winds down in order, and the status word says so."""
    bt = R.Batch([1500, 900], [200, 300], 8, 8, 128, 64, int8=int8, seed=7)
    assert P.sasq_device_status() == 0
    old = P.sasq_debug_set_wait_limit(0)
    try:
        attend(bt)
        status = P.sasq_device_status()
    finally:
        P.sasq_debug_set_wait_limit(-1)
    assert old == 1 << 31
    assert status == 5
    check(bt)


def test_a_view_of_one_head_or_one_page():
    """Dimensions of one entry have strides that say nothing."""
    for heads, n_pages in ((1, 3), (2, 1)):
        k = torch.randn((n_pages, 16, heads, 64), device="cuda").to(torch.bfloat16)
        odd = torch.as_strided(k, k.shape, [s if n > 1 else 3 for s, n in zip(k.stride(), k.shape)])
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        q = torch.randn((20, heads, 64), device="cuda").to(torch.bfloat16)
        outs = []
        for cache_k in (k, odd):
            cache = P.KVCache(cache_k, cache_k)
            batch = P.PagedBatch(i32([[n_pages - 1]]), i32([16]), i32([0, 20]), 20, 20, 16)
            out = torch.empty_like(q)
            ws = torch.empty(P.sasq_paged_attention_workspace(cache, batch, heads), dtype=torch.uint8, device="cuda")
            P.sasq_paged_attention(cache, batch, q, out, ws)
            outs.append(out)
        assert P.sasq_device_status() == 0 and torch.equal(outs[0], outs[1]) and (outs[0][:4] == 0).all()


@pytest.mark.parametrize("new", [1, 100])
def test_bad_factors_are_reported(new):
    for which in ("k_scale", "v_scale"):
        for wrong in (0.0, float("nan"), float("inf")):
            bt = R.Batch([200], [new], 4, 4, 64, 16, int8=True, seed=3)
            getattr(bt, which)[2] = wrong
            attend(bt)
            assert P.sasq_device_status() == 4


@pytest.mark.parametrize("new", [1, 100])
def test_negative_factors(new):
    bt = R.Batch([300, 200], [new] * 2, 4, 2, 128, 32, int8=True, seed=4)
    bt.k_scale[0] *= -1
    bt.v_scale[1] *= -1
    check(bt)


@pytest.mark.parametrize("new", [2, 150])
def test_loud_keys_out_of_sight(new):
    """Keys that a row must not see have logits far above all others (and are NaN for K): only the mask keeps them out."""
    bt = R.Batch([new + 40], [new], 4, 4, 128, 64, seed=5, tokens_first=True)
    last = new + 39
    page, row = int(bt.table[0, last // 64]), last % 64
    bt.k_host[page, row] = float("nan")
    bt.k.copy_(bt.k_host)
    out, lse = attend(bt)
    short = R.Batch([new + 40], [new], 4, 4, 128, 64, seed=5, tokens_first=True)
    want, want_lse, tol, lse_tol = R.attention(short, 128 ** -0.5, True)
    assert (np.abs(out.float().cpu().double().numpy() - want) <= tol)[:-1].all()
    assert (np.abs(lse.cpu().double().numpy() - want_lse) <= lse_tol)[:-1].all()


@pytest.mark.parametrize("new", [1, 3])
def test_more_heads_per_key_head_than_a_row_tile(new):
    for int8 in (False, True):
        check(R.Batch([90, 400], [new] * 2, 130, 1, 64, 16, int8=int8, seed=2))


@pytest.mark.parametrize("heads", [24, 48, 100, 128])
def test_groups_that_do_not_divide_a_row_tile(heads):
    check(R.Batch([500, 260], [40, 33], heads, 1, 64, 32, torch.float16, seed=heads))


def test_a_cache_without_pages():
    k = torch.empty((0, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    for new in (1, 30):
        cache = P.KVCache(k, k)
        batch = P.PagedBatch(torch.zeros((2, 1), dtype=torch.int32, device="cuda"), i32([0, 0]), i32([0, new, 2 * new]), 2 * new, new, 0)
        q = torch.randn((2 * new, 4, 64), device="cuda").to(torch.bfloat16)
        out, lse = torch.full_like(q, 7.0), torch.zeros((2 * new, 4), device="cuda")
        ws = torch.empty(P.sasq_paged_attention_workspace(cache, batch, 4), dtype=torch.uint8, device="cuda")
        P.sasq_paged_attention(cache, batch, q, out, ws, lse=lse)
        assert P.sasq_device_status() == 0 and (out == 0).all() and torch.isneginf(lse).all()
