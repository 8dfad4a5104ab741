"""Rotation and append: bit for bit what the definition gives in fp32 with one rounding per operation."""
import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu


def table(n, rot, seed=0):
    g = np.random.default_rng(seed)
    angle = g.uniform(0, 2 * np.pi, (n, rot // 2))
    return np.concatenate((np.cos(angle), np.sin(angle)), axis=1).astype(np.float32)


def codes(x, scale):
    inv = (np.float32(1.0) / scale.astype(np.float32)).astype(np.float32)
    return np.clip(np.rint((x * inv[:, None]).astype(np.float32)), -128, 127).astype(np.int8)


def run_case(lens, new, heads, kv_heads, dim, page, dtype, int8, rot, interleaved, tokens_first=False, with_q=True,
             in_place=False, pad_rows=0):
    bt = R.Batch(lens, new, heads, kv_heads, dim, page, dtype, int8, tokens_first, seed=dim + page, pad_rows=pad_rows)
    cache, batch = bt.handles(P)
    g = torch.Generator().manual_seed(1)
    qkv = (torch.randn((bt.T, heads + 2 * kv_heads, dim), generator=g) * 1.5).to(dtype)
    dev = qkv.cuda()
    cs = table(max(lens) + 3, rot) if rot else None
    q, k, v = dev[:, :heads], dev[:, heads:heads + kv_heads], dev[:, heads + kv_heads:]
    q_out = q if in_place else torch.full((bt.T, heads, dim), 7.0, dtype=dtype, device="cuda")
    P.sasq_rope_kv_append(cache, batch, q if with_q else None, k, v, q_out if with_q else None,
                          None if cs is None else torch.from_numpy(cs).cuda(), interleaved=interleaved)
    assert P.sasq_device_status() == 0
    host = qkv.float().numpy()
    want_k, want_v = bt.k_host.clone(), bt.v_host.clone()
    want_q = qkv[:, :heads].clone() if in_place else torch.full((bt.T, heads, dim), 7.0, dtype=dtype)
    for b, (l, n) in enumerate(zip(lens, new)):
        rows = np.arange(bt.starts[b], bt.starts[b] + n)
        pos = l - n + np.arange(n)
        want_q[rows[pos < 0]] = 0
        rows, pos = rows[pos >= 0], pos[pos >= 0]
        x = host[rows]
        turned = R.rotate(x, cs, pos, interleaved) if rot else x
        want_q[rows] = torch.from_numpy(turned[:, :heads]).to(dtype)
        page_of = torch.from_numpy(bt.table[b, pos // page].astype(np.int64))
        for want, y, f in ((want_k, turned[:, heads:heads + kv_heads], bt.k_scale), (want_v, x[:, heads + kv_heads:], bt.v_scale)):
            y = torch.from_numpy(codes(y, f.numpy())) if int8 else torch.from_numpy(y).to(dtype)
            want[page_of, torch.from_numpy(pos % page)] = y
    bits = (lambda t: t) if int8 else (lambda t: t.contiguous().view(torch.int16))
    assert torch.equal(bits(bt.k.cpu()), bits(want_k))
    assert torch.equal(bits(bt.v.cpu()), bits(want_v))
    if with_q:
        assert torch.equal(q_out.cpu().contiguous().view(torch.int16), want_q.view(torch.int16))


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (64, 64), (128, 64), (64, 16), (80, 48), (256, 256), (16, 16), (128, 0)])
def test_rotation_and_append(dim, rot, interleaved, dtype, int8):
    run_case([1, 40, 33, 200], [1, 40, 2, 77], 6, 2, dim, 16, dtype, int8, rot, interleaved)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("tokens_first", [True, False])
def test_pages_and_orders(page, tokens_first):
    lens = [page, page + 1, 2 * page - 1, 5]
    for int8 in (False, True):
        run_case(lens, [page, 2, page, 1], 4, 4, 64, page, torch.bfloat16, int8, 64, False, tokens_first)


def test_single_tokens_of_many_sequences():
    lens = [1 + (13 * i) % 70 for i in range(700)]
    run_case(lens, [1 if i % 5 else 0 for i in range(700)], 4, 1, 64, 16, torch.bfloat16, False, 64, False)


def test_without_q_in_place_padding_and_tokens_without_a_place():
    run_case([50, 9], [3, 4], 4, 2, 64, 16, torch.float16, False, 64, False, with_q=False)
    run_case([50, 9], [3, 4], 4, 2, 64, 16, torch.float16, True, 64, True, in_place=True)
    run_case([50, 9], [3, 4], 4, 2, 64, 16, torch.float16, False, 64, False, pad_rows=5)
    run_case([2, 0, 9], [6, 3, 4], 4, 2, 128, 16, torch.bfloat16, False, 128, False)


def test_large_and_one_by_one_agree():
    """A prompt appended at once and the same tokens appended one at a time leave the same cache."""
    n, K, D = 150, 3, 64
    bt = R.Batch([n], [n], 3, K, D, 32, torch.bfloat16, seed=3)
    cache, batch = bt.handles(P)
    x = torch.randn((n, 3 * K, D), device="cuda").to(torch.bfloat16)
    cs = torch.from_numpy(table(n, D)).cuda()
    q_all = torch.empty((n, K, D), dtype=torch.bfloat16, device="cuda")
    P.sasq_rope_kv_append(cache, batch, x[:, :K], x[:, K:2 * K], x[:, 2 * K:], q_all, cs)
    k_all, v_all = bt.k.clone(), bt.v.clone()
    bt.k.zero_(), bt.v.zero_()
    q_one = torch.empty((1, K, D), dtype=torch.bfloat16, device="cuda")
    starts = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for i in range(n):
        one = P.PagedBatch(batch.page_table, torch.tensor([i + 1], dtype=torch.int32, device="cuda"), starts, 1, 1, n)
        t = x[i:i + 1]
        P.sasq_rope_kv_append(cache, one, t[:, :K], t[:, K:2 * K], t[:, 2 * K:], q_one, cs)
        assert torch.equal(q_one[0], q_all[i])
    pos = np.arange(n)
    page, row = torch.from_numpy(bt.table[0, pos // 32].astype(np.int64)).cuda(), torch.from_numpy(pos % 32).cuda()
    assert torch.equal(bt.k[page, row], k_all[page, row]) and torch.equal(bt.v[page, row], v_all[page, row])


def test_places_outside_are_skipped_and_reported():
    bt = R.Batch([100, 100], [2, 2], 2, 2, 64, 16, seed=1)
    x = torch.randn((4, 6, 64), device="cuda").to(torch.bfloat16)
    q_out = torch.full((4, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    cs = torch.from_numpy(table(100, 64)).cuda()

    def call(cs):
        cache, batch = bt.handles(P)
        P.sasq_rope_kv_append(cache, batch, x[:, :2], x[:, 2:4], x[:, 4:], q_out, cs)
        return P.sasq_device_status()

    good = bt.table[0, 6]
    for wrong in (-1, 1 << 20):
        bt.table[0, 6] = wrong
        assert call(cs) == 7
        assert (q_out[:2] == 0).all() and not (q_out[2:] == 7).any()
    bt.table[0, 6] = good
    assert call(cs[:99].contiguous()) == 7                 # position 99 has no cosines
    bt.seq_lens[0] = 5000                                  # beyond the table
    assert call(cs) == 7
    bt.seq_lens[0] = 100
    assert call(cs) == 0


def test_bad_factor_is_reported():
    bt = R.Batch([10], [2], 2, 2, 64, 16, int8=True, seed=1)
    bt.k_scale[1] = 0.0
    cache, batch = bt.handles(P)
    x = torch.randn((2, 4, 64), device="cuda").to(torch.bfloat16)
    P.sasq_rope_kv_append(cache, batch, None, x[:, :2], x[:, 2:], None, None)
    assert P.sasq_device_status() == 4
