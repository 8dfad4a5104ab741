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

    A logit is the sum of q s c over the channels.  Either q s is taken as a multiple of 2^-22 of the row's largest, M, half a
    step off at most for each of n non-zero elements, and the sums are exact but for 8 roundings of 2^-24 of at most 16 A,
    A = sum |q s|; or q and s c are taken as 16-bit floats (exact while a row's elements lie within 2^16 of its largest, which
    these inputs do), and n additions are off by at most 2^-23 (the tensor cores may truncate) of 8 A each:
    e = max(8 n 2^-22 M + 2^-17 A, (n + 8) 2^-20 A) scale.  The second product is taken with c + 8: its fp32 sums add
    keys 2^-23 15 max(s) to what the other caches' bound allows."""
    out, lse, out_tol, lse_tol = R.attention(batch, scale, causal)
    q_all = batch.q_wide[:, :batch.heads].double().numpy()
    G = batch.heads // batch.kv_heads
    for b, (l, n) in enumerate(zip(batch.seq_lens, batch.new_lens)):
        rows = slice(int(batch.starts[b]), int(batch.starts[b]) + n)
        _, v = batch.keys(b)
        for c in range(batch.heads):
            s = used(batch.k_scale[c // G]).double().abs().numpy()
            nz = (q_all[rows, c] != 0).sum(axis=1)
            qs = np.abs(q_all[rows, c]) * s
            A = qs.sum(axis=1)
            e = np.maximum(8 * nz * 2.0 ** -22 * qs.max(axis=1, initial=0.0) + 2.0 ** -17 * A, (nz + 8) * 2.0 ** -20 * A) * abs(scale)
            big = np.abs(v[:, c // G]).max(initial=0.0)
            sv = used(batch.v_scale[c // G]).double().abs().numpy().max()
            lse_tol[rows, c] += e
            out_tol[rows, c] += (2 * e * big)[:, None] + (l + 8) * 2.0 ** -23 * 15 * sv
    return out, lse, out_tol, lse_tol
