"""The served attention block of examples/: a prompt in one pass, in chunks and token by token leave the same cache, bit for
bit, and outputs that agree to the rounding of the probabilities; and the block's attention matches a plain one."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("int8", [False, True])
def test_prompt_at_once_in_chunks_and_token_by_token(int8):
    import serve_attention as S
    block = S.AttentionBlock(hidden=512, heads=8, kv_heads=2, dim=64)
    n, cos_sin = 150, S.rotary_table(200, 64)
    x = torch.randn((2, n, 512), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    caches, outs, contexts = [], [], []
    for sizes in ([n], [100, 37, 13], [1] * n):
        pool = S.PagePool(block, 12, page=32, int8=int8)
        for seq in (0, 1):                                   # the same pages whatever the order of growth
            pool.room(seq, n)
        at, out, context = 0, torch.empty_like(x), torch.empty_like(x)
        steps = {m: S.Step(block, pool, [m, m], 200, cos_sin) for m in set(sizes)}
        for m in sizes:
            step = steps[m]
            step.x.copy_(x[:, at:at + m].reshape(-1, 512))
            at += m
            step.set_lengths([at, at])
            out[:, at - m:at] = step().view(2, m, 512)
            context[:, at - m:at] = step.ctx.view(2, m, 512)
        assert S.P.sasq_device_status() == 0
        caches.append((pool.k.clone(), pool.v.clone(), pool))
        outs.append(out)
        contexts.append(context)
    for k, v, _ in caches[1:]:
        assert torch.equal(k, caches[0][0]) and torch.equal(v, caches[0][1])
    # each context is off by u |out| + A (u + small), A = sum p |v| <= max |v|, u = 2^-8: two of them by twice that
    big = caches[0][1].float().abs().max().item() * (5.0 / 127 if int8 else 1.0)
    for c in contexts[1:]:
        assert (c.float() - contexts[0].float()).abs().max().item() <= 2 * 2 * (2.0 ** -8 + 2.0 ** -16) * big


def test_serving_loop_runs():
    import serve_attention as S
    prefill_ms, step_ms = S.serve(batch=3, prompt=200, steps=5, chunk=128, int8=True)
    assert prefill_ms > 0 and step_ms > 0
