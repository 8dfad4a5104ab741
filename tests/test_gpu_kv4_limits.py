"""The 4-bit cache and linear at their limits: offsets that pass 32 bits, the largest number of tokens, factors near the end of
fp32's range, calls on two streams and graphs at once, and a wait that runs out."""
import numpy as np
import pytest
import torch

import kv4_reference as R4
import paper_2512_14481_b200 as P
from test_gpu_kv4_append import run_case
from test_gpu_kv4_attention import check
from test_gpu_w4_linear import exact, problem, run

pytestmark = pytest.mark.gpu


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_clean():
    """The many-row kernel with a wait limit of zero cycles: it winds down in order, and the status word says so."""
    bt = R4.Batch([1500, 900], [200, 300], 8, 8, 128, 64, seed=7)
    assert P.sasq_device_status() == 0
    cache, batch = bt.handles(P)
    out = torch.empty((bt.T, 8, 128), dtype=bt.dtype, device="cuda")
    ws = torch.empty(P.sasq_paged_attention_workspace(cache, batch, 8), dtype=torch.uint8, device="cuda")
    P.sasq_debug_set_wait_limit(0)
    try:
        P.sasq_paged_attention(cache, batch, bt.q, out, ws)
        status = P.sasq_device_status()
    finally:
        P.sasq_debug_set_wait_limit(-1)
    assert status == 5
    check(bt)


@pytest.mark.parametrize("new", [1, 2, 50])
@pytest.mark.parametrize("by", [2.0 ** 104, 2.0 ** -60])
def test_far_value_factors(new, by):
    """Results of up to 2^109 are bf16 numbers."""
    bt = R4.Batch([150, 1, 90], [new, 1, new], 4, 2, 64, 16, torch.bfloat16, seed=4)
    bt.v_scale = bt.v_scale * by
    check(bt)


@pytest.mark.parametrize("tokens_first", [False, True])
@pytest.mark.parametrize("new", [1, 60])
def test_pages_behind_four_gigabytes(new, tokens_first):
    """The same sequence in the first pages of a pool and in its last ones, K and V in one pool of 4.5 GB, each in its own pages."""
    page, kv, dim, keys = 256, 8, 128, 1000
    pages = 4_500_000_000 // (page * kv * dim // 2)
    shape = (pages, page, kv, dim // 2) if tokens_first else (pages, kv, page, dim // 2)
    pool = torch.empty(shape, dtype=torch.uint8, device="cuda")
    assert pool.numel() > 1 << 32
    pool = pool if tokens_first else pool.transpose(1, 2)
    g = torch.Generator().manual_seed(new)
    fk, fv = (torch.rand((kv, dim), generator=g).cuda() + 0.2 for _ in range(2))
    k, v = (torch.randn((keys, kv, dim), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn((new, 2 * kv, dim), generator=g).to(torch.bfloat16).cuda()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    results = []
    for first in (0, pages - 8):
        # K's pages are 0 ... 3 of the eight, V's the other four: a view of the pool from four pages on
        n = pages - 4
        cache = P.KVCache(pool[:n], pool[4:], fk, fv)
        table = i32([[first + i if first == 0 else n - 4 + i for i in range(4)]])
        whole = P.PagedBatch(table, i32([keys]), i32([0, keys]), keys, keys, keys)
        P.sasq_rope_kv_append(cache, whole, None, k, v, None, None)
        last = P.PagedBatch(table, i32([keys]), i32([0, new]), new, new, keys)
        out, lse = torch.empty_like(q), torch.empty((new, 2 * kv), device="cuda")
        ws = torch.empty(max(16, P.sasq_paged_attention_workspace(cache, last, 2 * kv)), dtype=torch.uint8, device="cuda")
        P.sasq_paged_attention(cache, last, q, out, ws, lse=lse)
        at = int(table[0, 0])
        results.append((cache.k[at:at + 4].clone(), cache.v[at:at + 4].clone(), out, lse))
    assert P.sasq_device_status() == 0
    for i, (a, b) in enumerate(zip(*results)):
        if i < 2:
            a, b = a.transpose(1, 2).transpose(0, 1).flatten(1, 2), b.transpose(1, 2).transpose(0, 1).flatten(1, 2)
            a, b = a[:, :keys], b[:, :keys]
        assert torch.equal(a, b)
    inv = np.float32(1.0) / R4.used(fk.cpu()).numpy()
    want = np.clip(np.rint(k.float().cpu().numpy() * inv), -8, 7).astype(np.int8)
    stored = results[1][0].cpu().transpose(1, 2).transpose(0, 1).flatten(1, 2)[:, :keys]
    assert np.array_equal(R4.unpacked(stored).transpose(0, 1).numpy(), want)


@pytest.mark.parametrize("T", [1, 3, 12])
def test_weights_behind_four_gigabytes(T):
    N, K, group = (1 << 20) + 40, 8192 + 64, 64
    w = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda")
    assert w.numel() > 1 << 32
    scale = (torch.rand((N, K // group), device="cuda") + 0.1).to(torch.bfloat16)
    x = torch.randn((T, K), device="cuda").to(torch.bfloat16)
    y = torch.full((T, N), 7.0, dtype=torch.bfloat16, device="cuda")
    P.sasq_w4_linear(x, w, scale, y)
    assert P.sasq_device_status() == 0
    for rows in (slice(0, 40), slice(N // 2, N // 2 + 40), slice(N - 75, N)):
        want, tol = exact(x.cpu(), R4.unpacked(w[rows].cpu()), scale[rows].cpu(), None)
        assert (np.abs(y[:, rows].cpu().double().numpy() - want) <= tol).all()


def test_the_most_tokens():
    T = 1 << 19
    x, codes, scale, bias = problem(T, 20, 32, 32, torch.float16, bias=True)
    y = run(x, codes, scale, bias)
    for rows in (slice(0, 50), slice(T // 2 - 3, T // 2 + 50), slice(T - 50, T)):
        want, tol = exact(x[rows], codes, scale, bias)
        assert (np.abs(y[rows].double().numpy() - want) <= tol).all()


def test_two_streams_and_two_graphs_at_once():
    """Decode steps of two batches and linears, eager and replayed, side by side: each has its own workspace and result."""
    sides = []
    for seed in (1, 2):
        bt = R4.Batch([3000, 40, 700], [1, 1, 1], 16, 2, 128, 32, torch.float16, seed=seed)
        cache, batch = bt.handles(P)
        x, codes, scale, _ = problem(seed, 3000, 2048, 128, torch.float16)
        dev = [t.cuda() for t in (x, R4.packed(codes), scale)]
        out, y = torch.empty((bt.T, 16, 128), dtype=bt.dtype, device="cuda"), torch.empty((seed, 3000), dtype=bt.dtype, device="cuda")
        ws = torch.empty(P.sasq_paged_attention_workspace(cache, batch, 16), dtype=torch.uint8, device="cuda")

        def call(cache=cache, batch=batch, q=bt.q, out=out, ws=ws, dev=dev, y=y):
            P.sasq_paged_attention(cache, batch, q, out, ws)
            P.sasq_w4_linear(*dev, y)
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        sides.append((call, graph, out, y, out.clone(), y.clone(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for step in range(10):
        for call, graph, out, y, _, _, stream in sides:
            with torch.cuda.stream(stream):
                out.zero_()
                y.zero_()
                call() if step % 2 else graph.replay()
    torch.cuda.synchronize()
    assert P.sasq_device_status() == 0
    for _, _, out, y, want, want_y, _ in sides:
        assert torch.equal(out, want) and torch.equal(y, want_y)


def test_a_linears_wait_that_runs_out_is_reported_and_the_next_call_is_clean():
    """More than 16 tokens go through barriers; with a wait limit of zero cycles the kernel winds down, and the status word says so."""
    x, codes, scale, _ = problem(40, 6000, 4096, 64, torch.bfloat16)
    on = [t.cuda() for t in (x, R4.packed(codes), scale)]
    y = torch.empty((40, 6000), dtype=torch.bfloat16, device="cuda")
    assert P.sasq_device_status() == 0
    P.sasq_debug_set_wait_limit(0)
    try:
        P.sasq_w4_linear(*on, y)
        status = P.sasq_device_status()
    finally:
        P.sasq_debug_set_wait_limit(-1)
    assert status == 5
    P.sasq_w4_linear(*on, y)
    assert P.sasq_device_status() == 0
    want, tol = exact(x, codes, scale, None)
    assert (np.abs(y.cpu().double().numpy() - want) <= tol).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dim,rot", [(32, 32), (96, 32), (160, 0), (224, 224), (256, 128)])
def test_many_tokens_of_other_head_dims(dim, rot, in_place):
    """Many tokens go to blocks of 64 threads, which every head_dim shares out in its own way."""
    run_case([300, 0, 7, 350], [250, 0, 7, 340], 7, 3, dim, 32, torch.bfloat16, rot, dim == 96, in_place=in_place)
