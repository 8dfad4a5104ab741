"""Positions that the page table has no room for: the append skips them and touches nothing else, bit for bit."""
import numpy as np
import pytest
import torch

import paged_reference as R
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu

PAGE, PAGES = 16, 7
ROOM = PAGE * PAGES


def codes(x, scale):
    inv = (np.float32(1.0) / scale.astype(np.float32)).astype(np.float32)
    return np.clip(np.rint((x * inv[:, None]).astype(np.float32)), -128, 127).astype(np.int8)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("rot", [0, 64])
@pytest.mark.parametrize("length,new", [
    (ROOM + 1, 1),              # the first position without room, alone
    (ROOM + 1, 3),              # two tokens with a place, one without
    (ROOM + 8, 16),             # half of a page's tokens have a place
    (ROOM + 40, 3),             # none has
    (2 ** 31 - 1, 2),           # the largest length there is
    (-1, 1), (-2 ** 31, 5)])    # no length at all
def test_tokens_beyond_the_table_leave_the_cache_alone(length, new, rot, int8):
    heads, K, dim = 4, 2, 64
    bt = R.Batch([ROOM, 40], [new, 3], heads, K, dim, PAGE, int8=int8, seed=new, max_pages=PAGES)
    bt.seq_lens[0] = length
    cache, batch = bt.handles(P, max_seq=ROOM)
    qkv = torch.randn((bt.T, heads + 2 * K, dim), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    angle = np.random.default_rng(5).uniform(0, 2 * np.pi, (ROOM + 100, 32))
    cs = np.concatenate((np.cos(angle), np.sin(angle)), axis=1).astype(np.float32) if rot else None
    dev, q_out = qkv.cuda(), torch.full((bt.T, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    P.sasq_rope_kv_append(cache, batch, dev[:, :heads], dev[:, heads:heads + K], dev[:, heads + K:], q_out,
                          None if cs is None else torch.from_numpy(cs).cuda())
    assert P.sasq_device_status() == 7
    want_k, want_v = bt.k_host.clone(), bt.v_host.clone()
    want_q = torch.zeros((bt.T, heads, dim), dtype=torch.bfloat16)
    x_all = qkv.float().numpy()
    for b, (l, n) in enumerate(zip([length, 40], [new, 3])):
        pos = l - n + np.arange(n, dtype=np.int64)
        rows = bt.starts[b] + np.arange(n)
        has = (pos >= 0) & (pos < ROOM)
        pos, rows = pos[has], rows[has]
        x = x_all[rows]
        turned = R.rotate(x, cs, pos, False) if rot else x
        want_q[rows] = torch.from_numpy(turned[:, :heads]).to(torch.bfloat16)
        page, row = torch.from_numpy(bt.table[b, pos // PAGE].astype(np.int64)), torch.from_numpy(pos % PAGE)
        for want, y, f in ((want_k, turned[:, heads:heads + K], bt.k_scale), (want_v, x[:, heads + K:], bt.v_scale)):
            want[page, row] = torch.from_numpy(codes(y, f.numpy())) if int8 else torch.from_numpy(y).to(torch.bfloat16)
    bits = (lambda t: t) if int8 else (lambda t: t.contiguous().view(torch.int16))
    assert torch.equal(bits(bt.k.cpu()), bits(want_k))
    assert torch.equal(bits(bt.v.cpu()), bits(want_v))
    assert torch.equal(q_out.cpu().view(torch.int16), want_q.view(torch.int16))
