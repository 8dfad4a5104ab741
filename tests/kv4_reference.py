"""Inputs and 64-bit references for the 4-bit paged cache (numpy and torch on the host; nothing of the library is used)."""
import numpy as np
import torch

import paged_reference as R


def packed(codes):
    """int8 codes from -8 to 7 -> bytes, the even code in the low half."""
    u = (codes & 15).to(torch.uint8).unflatten(-1, (-1, 2))
    return u[..., 0] | u[..., 1] << 4


def unpacked(bytes_):
    u = torch.stack((bytes_ & 15, bytes_ >> 4), dim=-1).flatten(-2)
    return (u ^ 8).to(torch.int8) - 8


def used(factor):
    """A factor as the operators use it."""
    return factor.to(torch.bfloat16).float()


class Batch(R.Batch):
    """As the int8 batches of paged_reference, with 4-bit codes and a factor per KV head and channel.  Places that no key lives
    in hold -8 everywhere."""

    def __init__(self, seq_lens, new_lens, heads, kv_heads, dim, page, dtype=torch.bfloat16, tokens_first=False, seed=0, **kw):
        super().__init__(seq_lens, new_lens, heads, kv_heads, dim, page, dtype, True, tokens_first, seed, **kw)
        g = torch.Generator().manual_seed(seed + 1)
        self.k_scale, self.v_scale = ((torch.rand((kv_heads, dim), generator=g) + 0.5) / 4 for _ in range(2))
        loud = torch.rand((kv_heads, dim), generator=g) < 0.05
        self.k_scale = torch.where(loud, self.k_scale * 6, self.k_scale)
        self.set_codes(self.k_host >> 4, self.v_host >> 4, tokens_first)

    def set_codes(self, k, v, tokens_first=False):
        self.k_host, self.v_host = k, v
        self.k, self.v = (self._pool(packed(x), tokens_first) for x in (k, v))

    def keys(self, b):
        l = self.seq_lens[b]
        pos = np.arange(l)
        page, row = torch.from_numpy(self.table[b, pos // self.page].astype(np.int64)), torch.from_numpy(pos % self.page)
        return [(x[page, row].double() * used(f).double()).numpy() for x, f in ((self.k_host, self.k_scale), (self.v_host, self.v_scale))]


def attention(batch, scale, causal):
    """As paged_reference.attention, with the 4-bit cache's bounds.

    A logit is the sum of q s (c + 8) over the channels, each in two parts that are exact, less 8 sum q s.  With n non-zero
    elements of q that is at most 2 n additions, each off by at most 2^-23 (the tensor cores may truncate) of partial sums
    of at most 15 A, A = sum |q s| scale; the second sum and the difference add 2^-23 (n + 3) 8 A:
    e = (2 n 15 + 8 n + 64) 2^-23 A.  A product's own f16 parts are exact while the row's elements lie within 2^16 of its
    largest, which these inputs do.  The second product is taken with c + 8 too: its fp32 sums add keys 2^-23 15 max(s) to
    what the other caches' bound allows."""
    out, lse, out_tol, lse_tol = R.attention(batch, scale, causal)
    q_all = batch.q_wide[:, :batch.heads].double().numpy()
    G = batch.heads // batch.kv_heads
    for b, (l, n) in enumerate(zip(batch.seq_lens, batch.new_lens)):
        rows = slice(int(batch.starts[b]), int(batch.starts[b]) + n)
        _, v = batch.keys(b)
        for c in range(batch.heads):
            s = used(batch.k_scale[c // G]).double().abs().numpy()
            nz = (q_all[rows, c] != 0).sum(axis=1)
            e = (38 * nz + 64) * 2.0 ** -23 * (np.abs(q_all[rows, c]) @ s) * abs(scale)
            big = np.abs(v[:, c // G]).max(initial=0.0)
            sv = used(batch.v_scale[c // G]).double().abs().numpy().max()
            lse_tol[rows, c] += e
            out_tol[rows, c] += (2 * e * big)[:, None] + (l + 8) * 2.0 ** -23 * 15 * sv
    return out, lse, out_tol, lse_tol
