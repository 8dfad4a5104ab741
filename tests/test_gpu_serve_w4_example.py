"""The example's attention block served at 4 bits: linears, append and attention run together, over steps of several sizes, and
each of a step's results matches the 64-bit definition of its operator on what the one before it left."""
import os
import sys
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import kv4_reference as R4
import paged_reference as R
from test_gpu_kv4_append import codes
from test_gpu_w4_linear import UNIT, exact

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
HIDDEN, HEADS, KV_HEADS, DIM = 512, 8, 2, 64


def linear(block, name, x):
    w, s = (t.cpu() for t in block.weights[name])
    return exact(x.cpu(), R4.unpacked(w), s, None)


def near(got, want, tol):
    assert (np.abs(got.float().cpu().double().numpy() - want) <= tol).all()


def check_step(block, pool, step, lens, new, cos_sin):
    """lens: keys of each sequence after the step, which gave each `new` tokens."""
    T, pos = len(lens) * new, np.concatenate([np.arange(n - new, n) for n in lens])
    cs = cos_sin.cpu().numpy()
    # linears; q has been rotated in place, in fp32 (2 products and a sum, each rounded) and narrowed once more
    for name in ("k", "v"):
        near(getattr(step, name).reshape(T, -1), *linear(block, name, step.x))
    want, tol = (a.reshape(T, HEADS, DIM) for a in linear(block, "q", step.x))
    half = DIM // 2
    c, s = (a[pos][:, None].astype(np.float64) for a in (cs[:, :half], cs[:, half:]))
    a, b, ta, tb = want[..., :half], want[..., half:], tol[..., :half], tol[..., half:]
    turned = np.concatenate((a * c - b * s, b * c + a * s), axis=-1)
    off = np.concatenate((ta * np.abs(c) + tb * np.abs(s), tb * np.abs(c) + ta * np.abs(s)), axis=-1)
    size = np.tile(np.abs(a) + np.abs(b) + ta + tb, 2)
    u = UNIT[block.dtype]
    near(step.q, turned, (off + 2.0 ** -22 * size) * (1 + u) + u * np.abs(turned))
    # the cache, code by code
    table = step.table.cpu().numpy()
    page, row = np.concatenate([table[i, np.arange(n - new, n) // pool.page] for i, n in enumerate(lens)]), pos % pool.page
    for store, x, factor, turns in ((pool.k, step.k, pool.cache.k_scale, True), (pool.v, step.v, pool.cache.v_scale, False)):
        x = x.float().cpu().numpy()
        stored = R4.unpacked(store.cpu()).numpy()[page, row]
        assert np.array_equal(stored, np.asarray(codes(R.rotate(x, cs, pos, False) if turns else x, factor.cpu())))
    # attention, from the queries and the cache as they are
    kk, vv = (R4.unpacked(t.cpu()).double() for t in (pool.k, pool.v))

    def keys(i):
        at = np.arange(lens[i])
        pages, rows = torch.from_numpy(table[i, at // pool.page].astype(np.int64)), torch.from_numpy(at % pool.page)
        return [(t[pages, rows] * R4.used(f.cpu()).double()).numpy() for t, f in ((kk, pool.cache.k_scale), (vv, pool.cache.v_scale))]
    batch = SimpleNamespace(dtype=block.dtype, T=T, heads=HEADS, kv_heads=KV_HEADS, dim=DIM, q_wide=step.q.cpu(), seq_lens=lens,
                            new_lens=[new] * len(lens), starts=np.arange(len(lens) + 1) * new, keys=keys,
                            k_scale=pool.cache.k_scale.cpu(), v_scale=pool.cache.v_scale.cpu())
    want, _, tol, _ = R4.attention(batch, DIM ** -0.5, True)
    near(step.ctx3, want, tol)
    near(step.out, *linear(block, "o", step.ctx))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_steps_of_a_prompt(dtype):
    import serve_attention as S
    block = S.AttentionBlock(HIDDEN, HEADS, KV_HEADS, DIM, dtype=dtype, int4=True)
    cos_sin = S.rotary_table(200, DIM)
    pool = S.PagePool(block, 20, page=32, int4=True)
    g, at = torch.Generator().manual_seed(3), 0
    for new in (100, 17, 5, 1, 1, 2):
        step = S.Step(block, pool, [new] * 3, 200, cos_sin)
        step.x.copy_(torch.randn((3 * new, HIDDEN), generator=g).to(dtype))
        at += new
        step.set_lengths([at] * 3)
        step()
        assert S.P.sasq_device_status() == 0
        check_step(block, pool, step, [at] * 3, new, cos_sin)


def test_replayed_steps_of_one_token_on_another_stream():
    import serve_attention as S
    block = S.AttentionBlock(HIDDEN, HEADS, KV_HEADS, DIM, int4=True)
    cos_sin = S.rotary_table(200, DIM)
    pool = S.PagePool(block, 20, page=32, int4=True)
    step = S.Step(block, pool, [1, 1], 200, cos_sin)
    g, stream = torch.Generator().manual_seed(4), torch.cuda.Stream()
    step.x.zero_()
    step.set_lengths([1, 1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    with torch.cuda.graph(graph):
        step()
    for n in range(1, 70):
        step.x.copy_(torch.randn((2, HIDDEN), generator=g).to(block.dtype))
        step.set_lengths([n, n])
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.current_stream().wait_stream(stream)
        if n in (1, 2, 31, 32, 33, 69):
            check_step(block, pool, step, [n, n], 1, cos_sin)
    assert S.P.sasq_device_status() == 0


def test_serving_loop_runs():
    import serve_attention as S
    prefill_ms, step_ms = S.serve(batch=3, prompt=200, steps=5, chunk=128, int4=True)
    assert prefill_ms > 0 and step_ms > 0
