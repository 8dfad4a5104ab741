"""Attention: what lies in rows that no query owns has no part in a result, not in its last bit either.

An item of the many-row kernel has 256 rows, of which a sequence may fill fewer.  The others hold what shared memory held, or
the queries of the next sequence, or padding."""
import pytest
import torch

import kv4_reference as R4
import paged_reference as R
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu

KINDS = ("16-bit", "int8", "int4")
DTYPES = (torch.bfloat16, torch.float16)


def make(kind, lens, new, heads, kv_heads, dim, dtype, **kw):
    if kind == "int4":
        return R4.Batch(lens, new, heads, kv_heads, dim, 32, dtype, **kw)
    return R.Batch(lens, new, heads, kv_heads, dim, 32, dtype, kind == "int8", **kw)


def set_queries(bt, q):
    bt.q_wide, bt.q = q, q.cuda()[:, :bt.heads]


def attend(bt):
    cache, batch = bt.handles(P)
    out = torch.full((bt.T, bt.heads, bt.dim), 7.0, dtype=bt.dtype, device="cuda")
    lse = torch.full((bt.T, bt.heads), 7.0, device="cuda")
    ws = torch.empty(max(16, P.sasq_paged_attention_workspace(cache, batch, bt.heads)), dtype=torch.uint8, device="cuda")
    return lambda: P.sasq_paged_attention(cache, batch, bt.q, out, ws, lse=lse), out, lse


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,new", [(8, 50), (8, 37), (8, 20), (10, 60), (14, 90), (6, 100)])
def test_what_ran_before_does_not_show(heads, new, kind, dtype):
    """The same call behind one that fills every row with loud queries, and behind one that fills them with zeros."""
    target = make(kind, [700 - 9 * i for i in range(20)], [new] * 20, heads, 2, 128, dtype, seed=heads + new)
    before = make(kind, [300] * 24, [64] * 24, 32, 8, 128, dtype, seed=1)
    q = before.q_wide
    results = []
    for loud in (64.0, 0.0):
        set_queries(before, q * loud)
        fill, _, _ = attend(before)
        call, out, lse = attend(target)
        fill()
        call()
        results.append((out.clone(), lse.clone()))
    assert P.sasq_device_status() == 0
    (out, lse), (out0, lse0) = results
    assert torch.equal(out, out0) and torch.equal(lse, lse0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [1, 3, 37])
def test_other_sequences_queries_and_padding_do_not_show(new, kind, dtype):
    bt = make(kind, [900, 500, 640], [new] * 3, 8, 2, 128, dtype, seed=new, pad_rows=70)
    q = bt.q_wide.clone()
    results = []
    for other in (1.0, 40.0, float("nan")):
        changed = q.clone()
        changed[new:2 * new] = q[new:2 * new] * other      # the second sequence
        changed[3 * new:] = q[3 * new:] * other            # padding
        set_queries(bt, changed)
        call, out, lse = attend(bt)
        call()
        results.append((out.clone(), lse.clone()))
    assert P.sasq_device_status() == 0
    for out, lse in results[1:]:
        for mine in (slice(0, new), slice(2 * new, 3 * new), slice(3 * new, None)):
            assert torch.equal(out[mine], results[0][0][mine]) and torch.equal(lse[mine], results[0][1][mine])
    assert (results[0][0][3 * new:] == 7.0).all()
