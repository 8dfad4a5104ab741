"""Inputs and 64-bit references for the paged-cache operators (numpy only; nothing of the library is used here)."""
import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # half an ulp, relative


class Batch:
    """Ragged sequences over a shuffled page pool; every slot that no key lives in holds NaN (16-bit) or -128 (int8),
    and every table entry that no key needs holds -1."""

    def __init__(self, seq_lens, new_lens, heads, kv_heads, dim, page, dtype=torch.bfloat16, int8=False, tokens_first=False,
                 seed=0, max_pages=None, pad_rows=0, device="cuda", q_extra=0):
        g = torch.Generator().manual_seed(seed)
        self.seq_lens, self.new_lens = list(seq_lens), list(new_lens)
        self.heads, self.kv_heads, self.dim, self.page, self.dtype, self.int8 = heads, kv_heads, dim, page, dtype, int8
        need = [-(-l // page) for l in seq_lens]
        n_pages = max(1, sum(need) + 2)
        order = torch.randperm(n_pages, generator=g).tolist()
        width = max(1, max(need, default=0)) if max_pages is None else max_pages
        self.table = np.full((len(seq_lens), width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.starts = np.concatenate(([0], np.cumsum(new_lens))).astype(np.int32)
        self.T = int(self.starts[-1]) + pad_rows
        shape = (n_pages, page, kv_heads, dim)
        if int8:
            k = torch.randint(-128, 128, shape, generator=g, dtype=torch.int8)
            v = torch.randint(-128, 128, shape, generator=g, dtype=torch.int8)
            self.k_scale = (torch.rand(kv_heads, generator=g) + 0.5) / 64
            self.v_scale = (torch.rand(kv_heads, generator=g) + 0.5) / 64
        else:
            k, v = torch.randn(shape, generator=g).to(dtype), torch.randn(shape, generator=g).to(dtype)
            self.k_scale = self.v_scale = None
        used = torch.zeros((n_pages, page), dtype=torch.bool)
        for b, l in enumerate(seq_lens):
            for pos in range(0, l, page):
                used[self.table[b, pos // page], :min(page, l - pos)] = True
        k[~used] = -128 if int8 else float("nan")
        v[~used] = -128 if int8 else float("nan")
        # the rows of q lie further apart than their heads need (as in a fused projection's output)
        self.q_wide = torch.randn((self.T, heads + q_extra, dim), generator=g).to(dtype)
        self.k_host, self.v_host = k.clone(), v.clone()
        self.device = device
        self.k, self.v = (self._pool(x, tokens_first) for x in (k, v))
        self.q = self.q_wide.to(device)[:, :heads]

    def _pool(self, x, tokens_first):
        x = x.to(self.device)
        return x if tokens_first else x.transpose(1, 2).contiguous().transpose(1, 2)

    def handles(self, P, max_q=None, max_seq=None):
        to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(self.device)  # noqa: E731
        scales = (None, None) if not self.int8 else (self.k_scale.to(self.device), self.v_scale.to(self.device))
        cache = P.KVCache(self.k, self.v, *scales)
        batch = P.PagedBatch(to(self.table), to(np.array(self.seq_lens, dtype=np.int32)), to(self.starts), self.T,
                             max(self.new_lens, default=0) if max_q is None else max_q,
                             max(self.seq_lens, default=0) if max_seq is None else max_seq)
        return cache, batch

    def keys(self, b):
        """(k, v) of sequence b in 64 bits: [len, kv_heads, dim]."""
        l = self.seq_lens[b]
        pos = np.arange(l)
        page = self.table[b, pos // self.page]
        out = []
        for x, f in ((self.k_host, self.k_scale), (self.v_host, self.v_scale)):
            y = x[torch.from_numpy(page.astype(np.int64)), torch.from_numpy(pos % self.page)].double().numpy()
            out.append(y if f is None else y * f.double().numpy()[:, None])
        return out


def attention(batch, scale, causal):
    """(out, lse, bound on out, bound on lse) in 64 bits; rows that no sequence owns are NaN.

    Bounds.  A logit is an fp32 sum of dim exact products, so it is off by at most e = (dim + 3) 2^-24 sum |q k| scale; a
    probability's relative error is then e, plus 2^-20 for the exponential's approximation and the sum, plus its rounding
    to 16 bits (u; below the smallest normal fp16 number an absolute 2^-25 of a reference that is at most the row's
    maximum).  With A = sum_j p_j |v_j| that gives  u |out| + A (2 e + u + 2^-18) + keys 2^-25 max |v| for out, where
    2^-18 also covers the fp32 accumulation of the second product."""
    u = UNIT[batch.dtype]
    T, H, K, D = batch.T, batch.heads, batch.kv_heads, batch.dim
    G = H // K
    out, lse = np.full((T, H, D), np.nan), np.full((T, H), np.nan)
    out_tol, lse_tol = np.zeros((T, H, D)), np.zeros((T, H))
    q_all = batch.q_wide[:, :H].double().numpy()
    for b, (l, n) in enumerate(zip(batch.seq_lens, batch.new_lens)):
        k, v = batch.keys(b)
        rows = slice(int(batch.starts[b]), int(batch.starts[b]) + n)
        for c in range(H):
            q, kh, vh = q_all[rows, c], k[:, c // G], v[:, c // G]
            s = q @ kh.T * scale
            e = (np.abs(q) @ np.abs(kh).T * scale).max(axis=1, initial=0.0) * (D + 3) * 2.0 ** -24
            if causal:
                s = np.where(np.arange(l)[None, :] <= (l - n + np.arange(n))[:, None], s, -np.inf)
            m = s.max(axis=1, initial=-np.inf)
            p = np.exp(s - np.where(np.isfinite(m), m, 0.0)[:, None])
            total = p.sum(axis=1)
            with np.errstate(divide="ignore"):
                lse[rows, c] = m + np.log(total)
            p = p / np.where(total > 0, total, 1.0)[:, None]
            out[rows, c] = p @ vh
            A = p @ np.abs(vh)
            big = np.abs(vh).max(initial=0.0)
            out_tol[rows, c] = u * np.abs(out[rows, c]) + A * (2 * e[:, None] + u + 2.0 ** -18) + l * 2.0 ** -25 * big + 1e-30
            lse_tol[rows, c] = e + 2.0 ** -18 + np.abs(np.where(np.isfinite(lse[rows, c]), lse[rows, c], 0)) * 2.0 ** -22
    return out, lse, out_tol, lse_tol


def rotate(x, cos_sin, pos, interleaved):
    """x [n, heads, dim] at positions pos: the definition in fp32, each operation rounded once."""
    x = x.astype(np.float32).copy()
    rot = cos_sin.shape[1]
    half = rot // 2
    c, s = cos_sin[pos, :half].astype(np.float32)[:, None], cos_sin[pos, half:].astype(np.float32)[:, None]
    left, right = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    a, b = x[..., left].copy(), x[..., right].copy()
    x[..., left] = a * c - b * s
    x[..., right] = b * c + a * s
    return x
