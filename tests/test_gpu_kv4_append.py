"""Rotation and append to a 4-bit cache: bit for bit what the definition gives in fp32 with one rounding per operation."""
import numpy as np
import pytest
import torch

import kv4_reference as R4
import paged_reference as R
import paper_2512_14481_b200 as P
from test_gpu_paged_append import table

pytestmark = pytest.mark.gpu


def codes(x, factor):
    """x [n, heads, dim] fp32 -> int8 codes."""
    inv = np.float32(1.0) / R4.used(factor).numpy()
    return torch.from_numpy(np.clip(np.rint((x * inv).astype(np.float32)), -8, 7).astype(np.int8))


def run_case(lens, new, heads, kv_heads, dim, page, dtype, rot, interleaved, tokens_first=False, with_q=True, in_place=False,
             pad_rows=0, scale_of=None):
    bt = R4.Batch(lens, new, heads, kv_heads, dim, page, dtype, tokens_first, seed=dim + page, pad_rows=pad_rows)
    if scale_of is not None:
        bt.k_scale, bt.v_scale = scale_of(bt.k_scale), scale_of(bt.v_scale)
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
        at = torch.from_numpy(bt.table[b, pos // page].astype(np.int64)), torch.from_numpy(pos % page)
        want_k[at] = codes(turned[:, heads:heads + kv_heads], bt.k_scale)
        want_v[at] = codes(x[:, heads + kv_heads:], bt.v_scale)
    assert torch.equal(bt.k.cpu(), R4.packed(want_k))
    assert torch.equal(bt.v.cpu(), R4.packed(want_v))
    if with_q:
        assert torch.equal(q_out.cpu().contiguous().view(torch.int16), want_q.view(torch.int16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (64, 64), (128, 64), (64, 16), (96, 48), (256, 256), (32, 32), (128, 0)])
def test_rotation_and_append(dim, rot, interleaved, dtype):
    run_case([1, 40, 33, 200], [1, 40, 2, 77], 6, 2, dim, 16, dtype, rot, interleaved)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("tokens_first", [True, False])
def test_pages_and_orders(page, tokens_first):
    run_case([page, page + 1, 2 * page - 1, 5], [page, 2, page, 1], 4, 4, 64, page, torch.bfloat16, 64, False, tokens_first)


def test_single_tokens_of_many_sequences():
    lens = [1 + (13 * i) % 70 for i in range(700)]
    run_case(lens, [1 if i % 5 else 0 for i in range(700)], 4, 1, 64, 16, torch.bfloat16, 64, False)


def test_many_tokens():
    """More tokens than the device has blocks for at once, both ways of sharing a token's heads."""
    run_case([900, 1300], [900, 801], 8, 3, 128, 64, torch.float16, 128, False)
    run_case([40], [37], 64, 16, 128, 64, torch.bfloat16, 128, True)


def test_without_q_in_place_padding_and_tokens_without_a_place():
    run_case([50, 9], [3, 4], 4, 2, 64, 16, torch.float16, 64, False, with_q=False)
    run_case([50, 9], [3, 4], 4, 2, 64, 16, torch.float16, 64, True, in_place=True)
    run_case([50, 9], [3, 4], 4, 2, 64, 16, torch.float16, 64, False, pad_rows=5)
    run_case([2, 0, 9], [6, 3, 4], 4, 2, 128, 16, torch.bfloat16, 128, False)


@pytest.mark.parametrize("scale_of", [lambda f: -f, lambda f: f * 2.0 ** -100, lambda f: f * 2.0 ** 60, lambda f: f * 1e-3])
def test_factors(scale_of):
    """Negative, very small (everything saturates) and very large (all codes 0) factors."""
    run_case([33], [20], 2, 2, 64, 16, torch.bfloat16, 64, False, scale_of=scale_of)


def test_numbers_outside():
    """NaN gives the lowest code, infinities the end of their sign, as for the other quantizers."""
    bt = R4.Batch([3], [3], 1, 1, 32, 16, seed=1)
    cache, batch = bt.handles(P)
    x = torch.zeros((3, 2, 32), dtype=torch.bfloat16, device="cuda")
    x[0], x[1], x[2] = float("nan"), float("inf"), float("-inf")
    P.sasq_rope_kv_append(cache, batch, None, x[:, :1], x[:, 1:], None, None)
    assert P.sasq_device_status() == 0
    page = int(bt.table[0, 0])
    for t in (bt.k, bt.v):
        assert (t[page, 0].cpu() == 0x88).all() and (t[page, 1].cpu() == 0x77).all() and (t[page, 2].cpu() == 0x88).all()


def test_places_outside_are_skipped_and_reported():
    bt = R4.Batch([100, 100], [2, 2], 2, 2, 64, 16, seed=1)
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


@pytest.mark.parametrize("bad", [0.0, float("nan"), float("inf"), 1e-42, 3.4e38])
def test_bad_factor_is_reported(bad):
    """3.4e38 is finite and rounds to an infinite bfloat16."""
    bt = R4.Batch([10], [2], 2, 2, 64, 16, seed=1)
    x = torch.randn((2, 4, 64), device="cuda").to(torch.bfloat16)
    for name in ("k_scale", "v_scale"):
        cache, batch = bt.handles(P)
        getattr(cache, name)[1, 37] = bad
        P.sasq_rope_kv_append(cache, batch, None, x[:, :2], x[:, 2:], None, None)
        assert P.sasq_device_status() == 4
