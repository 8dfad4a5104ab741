"""The attention half of a W8A8 decoder layer, served: q / k / v linears, rotary positions and the append to a paged
cache, attention over the cache, o linear.  Prompts go through in chunks, then every sequence gets one token a step, the
step being replayed from a CUDA graph.  With --int4 the layer's weights have 4 bits with group factors, and the cache 4 bits
with a factor for each channel (its linears are made for decode steps: of a prompt's chunk they read the weights once for every
64 tokens).

    python examples/serve_attention.py [--batch 8] [--prompt 1000] [--steps 64] [--int8 | --int4]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2512_14481_b200 as P  # noqa: E402


class AttentionBlock:
    """Random frozen weights of one layer's four attention linears: int8 with static factors, or 4 bits with group factors."""

    def __init__(self, hidden=4096, heads=32, kv_heads=32, dim=128, dtype=torch.bfloat16, seed=0, int4=False, group=128):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.hidden, self.heads, self.kv_heads, self.dim, self.dtype = hidden, heads, kv_heads, dim, dtype
        self.int4, self.weights = int4, {}
        for name, n, k in (("q", heads * dim, hidden), ("k", kv_heads * dim, hidden), ("v", kv_heads * dim, hidden),
                           ("o", hidden, heads * dim)):
            w = torch.randn((n, k), generator=gen, device="cuda") * k ** -0.5
            if int4:
                w_int = torch.empty((n, k // 2), dtype=torch.uint8, device="cuda")
                w_scale = torch.empty((n, k // group), dtype=dtype, device="cuda")
                P.sasq_quantize_weight_w4(w, w_int, w_scale)
            else:
                w_int = torch.empty((n, k), dtype=torch.int8, device="cuda")
                w_scale = torch.empty(n, device="cuda")
                P.sasq_quantize_weight(w, w_int, w_scale)
            self.weights[name] = (w_int, w_scale)
        self.x_scale = torch.tensor([4.0 / 127], device="cuda")            # static factors, as learned
        self.o_scale = torch.tensor([2.0 / 127], device="cuda")

    def linears(self, problems):
        """One call for independent linears: (x, name, factor, y) each; returns a function that submits them."""
        if self.int4:
            def submit():
                for x, name, _, y in problems:
                    P.sasq_w4_linear(x, *self.weights[name], y)
            return submit
        table = P.LinearProblems([(x, *self.weights[name], factor, y) for x, name, factor, y in problems])
        shapes = [(x.shape[0], y.shape[1], x.shape[1]) for x, _, _, y in problems]
        ws = torch.empty(P.sasq_static_w8a8_linear_multi_workspace(shapes), dtype=torch.uint8, device="cuda")
        return lambda: P.sasq_static_w8a8_linear_multi(table, ws)


class PagePool:
    """Pages of one layer's cache and which sequence has which."""

    def __init__(self, block, pages, page=64, int8=False, int4=False):
        shape = (pages, block.kv_heads, page, block.dim // 2 if int4 else block.dim)       # heads first: a head's rows lie together
        dt = torch.uint8 if int4 else torch.int8 if int8 else block.dtype
        self.k = torch.zeros(shape, dtype=dt, device="cuda").transpose(1, 2)
        self.v = torch.zeros(shape, dtype=dt, device="cuda").transpose(1, 2)
        factors = (None, None)
        if int4:                                                           # static factors, as learned: one for each channel
            factors = [torch.full((block.kv_heads, block.dim), 3.0 / 7, device="cuda") for _ in range(2)]
        elif int8:
            factors = [torch.full((block.kv_heads,), 5.0 / 127, device="cuda") for _ in range(2)]
        self.cache = P.KVCache(self.k, self.v, *factors)
        self.page, self.free, self.owned = page, list(range(pages)), {}

    def room(self, seq, keys):
        """Gives the sequence enough pages for `keys` keys; returns all of its pages."""
        mine = self.owned.setdefault(seq, [])
        while len(mine) * self.page < keys:
            mine.append(self.free.pop())
        return mine


class Step:
    """One pass of `new[i]` tokens for sequence i, all buffers and tables in place; call it, or capture it in a graph.
    The lengths and page tables are device tensors: `set_lengths` moves a replayed step on."""

    def __init__(self, block, pool, new, max_keys, cos_sin, hidden_in=None):
        self.block, self.pool, self.new, T = block, pool, list(new), sum(new)
        B, D = len(new), block.dim
        max_pages = -(-max_keys // pool.page)
        self.table = torch.zeros((B, max_pages), dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        starts = torch.tensor([0] + list(torch.tensor(self.new).cumsum(0)), dtype=torch.int32, device="cuda")
        self.x = hidden_in if hidden_in is not None else torch.empty((T, block.hidden), dtype=block.dtype, device="cuda")
        buf = lambda n: torch.empty((T, n * D), dtype=block.dtype, device="cuda")  # noqa: E731
        q, k, v, self.ctx = buf(block.heads), buf(block.kv_heads), buf(block.kv_heads), buf(block.heads)
        self.out = torch.empty((T, block.hidden), dtype=block.dtype, device="cuda")
        self.batch = P.PagedBatch(self.table, self.lens, starts, T, max(new), max_keys)
        self.qkv = block.linears([(self.x, "q", block.x_scale, q), (self.x, "k", block.x_scale, k), (self.x, "v", block.x_scale, v)])
        self.o = block.linears([(self.ctx, "o", block.o_scale, self.out)])
        self.q, self.k, self.v = q.view(T, -1, D), k.view(T, -1, D), v.view(T, -1, D)
        self.ctx3, self.cos_sin = self.ctx.view(T, -1, D), cos_sin
        ws = P.sasq_paged_attention_workspace(pool.cache, self.batch, block.heads)
        self.ws = torch.empty(max(ws, 16), dtype=torch.uint8, device="cuda")

    def set_lengths(self, lengths):
        """Keys of each sequence after this step."""
        for b, n in enumerate(lengths):
            pages = self.pool.room(b, n)
            self.table[b, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        self.lens.copy_(torch.tensor(lengths, dtype=torch.int32))

    def __call__(self):
        self.qkv()
        P.sasq_rope_kv_append(self.pool.cache, self.batch, self.q, self.k, self.v, self.q, self.cos_sin)
        P.sasq_paged_attention(self.pool.cache, self.batch, self.q, self.ctx3, self.ws)
        self.o()
        return self.out


def rotary_table(positions, dim, base=10000.0):
    angle = torch.arange(positions, device="cuda")[:, None] * base ** (-torch.arange(0, dim, 2, device="cuda").double() / dim)
    return torch.cat((angle.cos(), angle.sin()), dim=1).float()


def serve(batch=8, prompt=1000, steps=64, chunk=512, int8=False, int4=False):
    """Prefills `batch` prompts chunk by chunk and decodes `steps` tokens; returns device times in ms (prefill, per step)."""
    block = AttentionBlock(int4=int4)
    max_keys = prompt + steps
    pool = PagePool(block, batch * -(-max_keys // 64) + 1, int8=int8, int4=int4)
    cos_sin = rotary_table(max_keys, block.dim)
    begin, mid, end = (torch.cuda.Event(enable_timing=True) for _ in range(3))
    sizes = [min(chunk, prompt - at) for at in range(0, prompt, chunk)]
    prefill = {n: Step(block, pool, [n] * batch, max_keys, cos_sin) for n in set(sizes)}
    decode = Step(block, pool, [1] * batch, max_keys, cos_sin)
    for s in (*prefill.values(), decode):
        s.x.normal_()
    decode.set_lengths([1] * batch)
    decode()                                                             # one-time set-up stays outside the graph
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode()
    begin.record()
    at = 0
    for n in sizes:
        at += n
        prefill[n].set_lengths([at] * batch)
        prefill[n]()
    mid.record()
    for i in range(steps):
        decode.set_lengths([prompt + i + 1] * batch)
        graph.replay()
    end.record()
    end.synchronize()
    status = P.sasq_device_status()
    if status != 0:
        raise P.SasqError(status, "serve")
    return begin.elapsed_time(mid), mid.elapsed_time(end) / max(1, steps)


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--steps", type=int, default=64)
    bits = ap.add_mutually_exclusive_group()
    bits.add_argument("--int8", action="store_true", help="an int8 cache")
    bits.add_argument("--int4", action="store_true", help="4-bit weights and a 4-bit cache")
    a = ap.parse_args()
    for _ in range(2):                                                   # the second round is warm
        prefill_ms, step_ms = serve(a.batch, a.prompt, a.steps, int8=a.int8, int4=a.int4)
    print(f"prefill {a.batch} x {a.prompt} tokens: {prefill_ms:.2f} ms; decode step of {a.batch}: {step_ms * 1000:.0f} us")
