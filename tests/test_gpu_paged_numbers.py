"""Numbers at the ends of their ranges: keys that count for little one by one, NaN in a query, factors that vanish."""
import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu


def attend(bt, scale=None):
    cache, batch = bt.handles(P)
    out = torch.full((bt.T, bt.heads, bt.dim), 7.0, dtype=bt.dtype, device="cuda")
    lse = torch.full((bt.T, bt.heads), 7.0, device="cuda")
    ws = torch.full((max(16, P.sasq_paged_attention_workspace(cache, batch, bt.heads)),), 255, dtype=torch.uint8, device="cuda")
    P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse, scale=scale)
    assert P.sasq_device_status() == 0
    return out.float().cpu().double().numpy(), lse.cpu().double().numpy()


def tail_bounds(bt, out_tol):
    """paged_reference.attention's bound with its absolute term taken to what 16-bit probabilities have to give: they
    are rounded against a reference that leaves the row's largest at 2^7 or more, so a probability below f16's normal
    range is off by at most 2^-25 / 2^7 of the row's largest.  An output below the normal range has 2^-25 of its own."""
    for b, l in enumerate(bt.seq_lens):
        _, v = bt.keys(b)
        rows = slice(int(bt.starts[b]), int(bt.starts[b + 1]))
        for c in range(bt.heads):
            big = np.abs(v[:, c // (bt.heads // bt.kv_heads)]).max(initial=0.0)
            out_tol[rows, c] += l * big * (2.0 ** -32 - 2.0 ** -25) + 2.0 ** -25
    return out_tol


@pytest.mark.parametrize("below", [20, 26, 30])
@pytest.mark.parametrize("dtype,int8", [(torch.float16, False), (torch.float16, True), (torch.bfloat16, True)])
@pytest.mark.parametrize("new,count", [(1, 200), (3, 100), (70, 60), (1, 3)])
def test_one_loud_key_and_many_faint_ones(new, count, dtype, int8, below):
    """The first key has nearly all of a row's weight and a value of zero: the result is what the others add up to, each
    2^-below of the first's.  (`count` sequences, so that no block has a part of the keys without the loud one.)"""
    lens = [900 + 7 * (i % 11) for i in range(count)]
    bt = R.Batch(lens, [new] * count, 4, 1, 64, 64, dtype, int8, tokens_first=True, seed=below)
    g = torch.Generator().manual_seed(below)
    k, v = torch.randn(bt.k_host.shape, generator=g), torch.rand(bt.v_host.shape, generator=g) * 6 + 6
    loud = below * np.log(2.0) / 8.0                               # 64 queries' elements of one, scale 1 / 8
    if int8:
        bt.k_scale, bt.v_scale = torch.full((1,), loud / 100), torch.full((1,), 0.1)
        k, v = k.clamp(-1, 1).round(), (v * 10).round()
    else:
        k = k * 0.03
    for b in range(count):
        page = int(bt.table[b, 0])
        k[page, 0], v[page, 0] = (100.0 if int8 else loud), 0.0
    bt.k_host, bt.v_host = k.to(bt.k_host.dtype), v.to(bt.v_host.dtype)
    bt.k.copy_(bt.k_host), bt.v.copy_(bt.v_host)
    bt.q_wide = torch.ones_like(bt.q_wide)
    bt.q.copy_(bt.q_wide)
    out, lse = attend(bt)
    want, want_lse, tol, lse_tol = R.attention(bt, 0.125, True)
    assert (np.abs(want) > 0).all()
    assert (np.abs(out - want) <= tail_bounds(bt, tol)).all()
    assert (np.abs(lse - want_lse) <= lse_tol).all()


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("new,count", [(1, 2), (1, 60), (12, 2), (12, 60), (70, 2), (70, 60)])
def test_nan_in_a_query_shows_in_its_own_row_only(new, count, dtype, int8):
    """A NaN is not a row without keys: out and lse of that (token, head) are NaN, all others are what they were."""
    lens = [new + 9 * i for i in range(count)]
    bt = R.Batch(lens, [new] * count, 4, 2, 64, 16, dtype, int8, seed=count)
    want, want_lse, tol, lse_tol = R.attention(bt, 0.125, True)
    hit = np.zeros((bt.T, 4), dtype=bool)
    for t, h in ((0, 1), (bt.T // 2, 3), (bt.T - 1, 0)):
        hit[t, h] = True
        bt.q[t, h, 5 * h] = float("nan")
    out, lse = attend(bt)
    assert np.isnan(out[hit]).all() and np.isnan(lse[hit]).all()
    assert (np.abs(out - want) <= tol)[~hit].all()
    assert (np.abs(lse - want_lse) <= lse_tol)[~hit].all()


@pytest.mark.parametrize("factor", [1e-20, 1e-30, -1e-30])
@pytest.mark.parametrize("new", [1, 12, 70])
def test_a_scale_and_a_factor_whose_product_vanishes(new, factor):
    """All logits are zero to fp32: every key that a row sees counts the same."""
    bt = R.Batch([new, 300], [new] * 2, 4, 4, 64, 16, int8=True, seed=new)
    bt.k_scale[:] = factor
    out, lse = attend(bt, scale=0.0)
    want, want_lse, tol, lse_tol = R.attention(bt, 0.0, True)
    assert (np.abs(out - want) <= tol).all()
    assert (np.abs(lse - want_lse) <= lse_tol).all()
