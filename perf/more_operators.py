"""The operators of a decoder layer served at 4 bits: what is run, on which sizes, and what each pass has to move.

Three operators: `append` (rotary positions on q and k, k and v appended to a paged cache of 4-bit codes), `attend`
(attention of the new tokens of a batch of sequences over that cache) and `linear` (few tokens through a linear layer with
4-bit weights and group factors).  Each has a plain form in elementary torch operations on fp32 values, and the framework's
own calls (where `own` is true)."""
import math
import random

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------------
def _paged(op, name=None, dt="bf16", heads=32, kv_heads=32, dim=128, page=16, batch=1, ctx=(0, 0), new=(1, 1), causal=True,
           layout="heads", style="half", rot=None):
    """ctx: tokens that the cache holds before the new ones, from the shortest to the longest sequence; new: new tokens."""
    c = {"op": op, "dt": dt, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "batch": batch,
         "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": new[0], "new_hi": new[1], "layout": layout}
    if op == "append":
        c["style"] = style
        c["rot"] = dim if rot is None else rot
    else:
        c["causal"] = causal
    return dict(c, name=name) if name else c


def _linear(name=None, dt="bf16", tokens=1, n=4096, k=4096, group=128, bias=False):
    c = {"op": "linear", "dt": dt, "tokens": tokens, "n": n, "k": k, "group": group, "bias": bias}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's next token in a LLaMA-2-7B-shaped layer, a new conversation: all latency
        _paged("append", "append one token", ctx=(100, 100)),
        # a decode step of a full batch with grouped heads, conversations just begun
        _paged("append", "append decode 128", kv_heads=8, batch=128, ctx=(1, 77), page=32),
        # chunks of prompts of a 13B-shaped layer with grouped heads, fp16, interleaved pairs on half of a head
        _paged("append", "append prompts fp16", dt="fp16", heads=40, kv_heads=8, batch=3, ctx=(0, 77), new=(1111, 2099), page=64,
               layout="tokens", style="pairs", rot=64),
        # one user's next token, LLaMA-2-7B-shaped, about a thousand tokens in
        _paged("attend", "decode one", ctx=(1000, 1000)),
        # a decode step of a batch of ragged conversations, grouped heads
        _paged("attend", "decode 64 ragged", kv_heads=8, batch=64, ctx=(30, 4500), page=32),
        # long documents, a few readers: what a 4-bit cache is for
        _paged("attend", "decode long", kv_heads=8, batch=8, ctx=(8000, 32000), page=64),
        # a draft's seven tokens checked at once, heads of 64, fp16, odd group of five
        _paged("attend", "verify 7 fp16", dt="fp16", heads=40, kv_heads=8, dim=64, batch=16, ctx=(100, 3000), new=(7, 7),
               layout="tokens"),
        # a chunk of a long prompt: the largest
        _paged("attend", "chunk 1024", kv_heads=8, ctx=(15000, 15000), new=(1024, 1024), page=128),
        # the output projection of one user's next token, LLaMA-2-7B-shaped: mostly latency
        _linear("linear one token"),
        # gate and up projections of a 7B-shaped layer as one matrix, one token, fp16
        _linear("linear one token wide fp16", dt="fp16", n=22016, k=4096),
        # down projection of a 13B-shaped layer, a draft's seven tokens, groups of 64, with a bias
        _linear("linear seven tokens deep", tokens=7, n=5120, k=13824, group=64, bias=True),
        # a batch of 61 sequences through q, k and v of a layer with grouped heads, groups of 32, fp16
        _linear("linear batch of 61 fp16", dt="fp16", tokens=61, n=6144, k=4096, group=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("append", "attend", "attend", "linear", "linear"))
        dt = rng.choice(("bf16", "bf16", "fp16"))
        if op == "linear":
            group = rng.choice((32, 64, 128, 128))
            c = _linear(dt=dt, tokens=_log(rng, 1, 64), n=_log(rng, 200, 28000), k=group * max(1, _log(rng, 200, 14000) // group),
                        group=group, bias=rng.random() < 0.3)
            if work(c)["bytes"] <= 6e7:
                return c
            continue
        group = rng.choice((1, 1, 2, 3, 4, 5, 7, 8))
        kv_heads = rng.choice((1, 2, 4, 5, 8, 8, 16, 32, 40))
        dim = rng.choice((64, 128, 128))
        kind = rng.choice(("decode", "few", "chunk", "prompt"))
        batch = _log(rng, 1, 128) if kind == "decode" else _log(rng, 1, 32) if kind == "few" else _log(rng, 1, 12)
        hi = _log(rng, 1, 32000) if kind != "prompt" and op == "attend" else _log(rng, 1, 200)
        new_hi = 1 if kind == "decode" else rng.randint(2, 16) if kind == "few" else _log(rng, 17, 1500) if kind == "chunk" \
            else _log(rng, 100, 4096)
        new_lo = 1 if kind == "decode" else rng.randint(1, new_hi)
        c = _paged(op, dt=dt, heads=group * kv_heads, kv_heads=kv_heads, dim=dim, page=rng.choice((16, 32, 64, 128)),
                   batch=batch, ctx=(rng.randint(0, hi), hi), new=(new_lo, new_hi), causal=rng.random() < 0.85,
                   layout=rng.choice(("heads", "tokens")), style=rng.choice(("half", "half", "pairs")),
                   rot=rng.choice((dim, dim, dim // 2)))
        if c["heads"] > 64:
            continue
        lens, new = _lengths(c)
        w, longest, most = work(c), max(lens), max(new)
        if op == "append" and w["bytes"] <= 1.4e8 and sum(lens) * kv_heads * dim <= 1 << 23:
            return c
        if op == "attend" and w["flops"] <= 2.6e11 and batch * longest * kv_heads * dim <= 1 << 29 \
                and batch * c["heads"] * most * longest <= 2 ** 31:
            return c


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, in a fixed shuffled order."""
    v = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]
    random.Random(n).shuffle(v)
    return v


def _lengths(case):
    """(keys in the cache with the new ones, new tokens) of each sequence: by the case alone."""
    n = case["batch"]
    new = _spread(case["new_lo"], case["new_hi"], n)
    ctx = _spread(case["ctx_lo"], case["ctx_hi"], n)[::-1]
    return [a + b for a, b in zip(ctx, new)], new


def _pairs(case):
    """Query-key pairs that the mask leaves, of one head."""
    lens, new = _lengths(case)
    if not case["causal"]:
        return sum(l * m for l, m in zip(lens, new))
    return sum(m * (l - m) + m * (m + 1) // 2 for l, m in zip(lens, new))


def work(case):
    if case["op"] == "linear":
        T, N, K = case["tokens"], case["n"], case["k"]
        return {"bytes": N * K // 2 + 2 * N * (K // case["group"]) + 2 * T * K + 2 * T * N + (2 * N if case["bias"] else 0),
                "flops": 2 * T * N * K}
    lens, new = _lengths(case)
    T, D, H, K = sum(new), case["dim"], case["heads"], case["kv_heads"]
    factors = 2 * K * D * 4
    if case["op"] == "append":
        places = len({p for l, m in zip(lens, new) for p in range(l - m, l)})
        return {"bytes": T * (H * D * 4 + K * D * 5) + places * case["rot"] * 4 + factors, "flops": 3 * T * (H + K) * case["rot"]}
    return {"bytes": sum(lens) * K * D + T * H * (D * 4 + 4) + factors, "flops": 4 * D * H * _pairs(case)}


# ---------------------------------------------------------------------------------------------------------------------
# the inputs
# ---------------------------------------------------------------------------------------------------------------------
def _values(shape, dt, gen, wide=0.02, by=4.0):
    """Normal values with a few louder channels, as projections of a decoder layer have them."""
    x = torch.randn(shape, generator=gen, device=DEVICE)
    loud = (torch.rand(shape[-2:], generator=gen, device=DEVICE) < wide).float() * (by - 1) + 1
    return x.mul_(loud).to(dt)


def _packed(codes):
    """Codes from -8 to 7, two to a byte: the even one in the low half."""
    pairs = (codes & 15).to(torch.uint8).unflatten(-1, (-1, 2))
    return pairs[..., 0] | pairs[..., 1] << 4


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = DTYPES[case["dt"]]
    if case["op"] == "linear":
        return _prepare_linear(case, gen, dt)
    lens, new = _lengths(case)
    P, D, H, K = case["page"], case["dim"], case["heads"], case["kv_heads"]
    T, B = sum(new), len(lens)
    need = [-(-l // P) for l in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.zeros((B, max(need)), dtype=torch.int32, device=DEVICE)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    # keys and values of all pages in one pool [keys / values, pages, ...], with what earlier requests left in it; the
    # static factor of a channel lets its largest fifth saturate
    pool, factor = [], []
    for _ in range(2):
        x = _values((n_pages, P, K, D), torch.float32, gen)
        f = x.abs().amax(dim=(0, 1)) * (0.8 / 7)
        s = f.to(torch.bfloat16).float()
        x = _packed(torch.clamp(torch.round(x / s), -8, 7).to(torch.int8))
        pool.append(x.transpose(1, 2) if case["layout"] == "heads" else x)
        factor.append(f)
    pool = torch.stack([x.contiguous() for x in pool])
    if case["layout"] == "heads":
        pool = pool.transpose(2, 3)
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    s = {"case": case, "pool": pool, "k": pool[0], "v": pool[1], "k_scale": factor[0], "v_scale": factor[1], "table": table,
         "lens": torch.tensor(lens, dtype=torch.int32, device=DEVICE),
         "starts": torch.tensor(starts, dtype=torch.int32, device=DEVICE), "longest": max(lens), "most": max(new), "T": T}
    if case["op"] == "append":
        # the three projections' outputs lie side by side in one buffer, as one fused linear leaves them
        s["qkv"] = _values((T, H + 2 * K, D), dt, gen)
        rot = case["rot"]
        angle = torch.arange(max(lens), device=DEVICE, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, rot, 2, device=DEVICE, dtype=torch.float64) / rot)
        s["cos_sin"] = torch.cat((angle.cos(), angle.sin()), dim=1).float()
        s["q_out"] = torch.empty((T, H, D), dtype=dt, device=DEVICE)
        # what a byte of the cache stands for, and the factors of its two codes, to read the cache back with
        codes = (torch.arange(16, device=DEVICE) + 8) % 16 - 8
        s["meaning"] = torch.stack((codes.repeat(16), codes.repeat_interleave(16)), dim=1).float()
        s["factors"] = torch.stack(factor).to(torch.bfloat16).float()[:, None, None]
    else:
        s["q"] = (_values((T, H, D), torch.float32, gen) * 1.5).to(dt)
        s["out"] = torch.empty((T, H, D), dtype=dt, device=DEVICE)
        s["lse"] = torch.empty((T, H), dtype=torch.float32, device=DEVICE)
    if own:  # the handles and the scratch memory that a serving loop keeps over its steps
        import paper_2512_14481_b200 as P_
        s["lib"] = P_
        s["cache"] = P_.KVCache(s["k"], s["v"], *factor)
        s["batch"] = P_.PagedBatch(table, s["lens"], s["starts"], T, s["most"], s["longest"])
        if case["op"] == "attend":
            s["ws"] = torch.empty(P_.sasq_paged_attention_workspace(s["cache"], s["batch"], H), dtype=torch.uint8, device=DEVICE)
    return s


def _prepare_linear(case, gen, dt):
    T, N, K, G = case["tokens"], case["n"], case["k"], case["group"]
    w = torch.randn((N, K // G, G), generator=gen, device=DEVICE).mul_(0.02)
    scale = (w.abs().amax(dim=2, keepdim=True) / 7).to(dt)
    codes = torch.clamp(torch.round(w / scale.float()), -8, 7).to(torch.int8)
    s = {"case": case, "x": _values((T, 1, K), dt, gen, wide=0.01, by=20.0).view(T, K), "w": _packed(codes.view(N, K)),
         "w_scale": scale.view(N, K // G), "y": torch.empty((T, N), dtype=dt, device=DEVICE), "bias": None}
    if case["bias"]:
        s["bias"] = torch.randn((N,), generator=gen, device=DEVICE).mul_(0.5).to(dt)
    if own:
        import paper_2512_14481_b200 as P_
        s["lib"] = P_
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if case["op"] == "linear":
        if own:
            s["lib"].sasq_w4_linear(s["x"], s["w"], s["w_scale"], s["y"], bias=s["bias"])
            return s["y"]
        return _linear_plain(s)
    if case["op"] == "append":
        H, K = case["heads"], case["kv_heads"]
        q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + K], s["qkv"][:, H + K:]
        if own:
            s["lib"].sasq_rope_kv_append(s["cache"], s["batch"], q, k, v, s["q_out"], s["cos_sin"],
                                         interleaved=case["style"] == "pairs")
            q_out = s["q_out"]
        else:
            q_out = _append_plain(s, q, k, v)
        values = s["meaning"][s["pool"].int()].flatten(-2).mul_(s["factors"])
        return {"q": q_out, "kv": values}
    if own:
        s["lib"].sasq_paged_attention(s["cache"], s["batch"], s["q"], s["out"], s["ws"], lse=s["lse"],
                                      scale=case["dim"] ** -0.5, causal=case["causal"])
        return {"out": s["out"], "lse": s["lse"]}
    return _attend_plain(s)


def _unpacked(bytes_):
    """fp32 codes of packed ones."""
    pairs = torch.stack((bytes_ & 15, bytes_ >> 4), dim=-1).flatten(-2)
    return ((pairs ^ 8).to(torch.int8) - 8).float()


def _linear_plain(s):
    case = s["case"]
    T, N, K, G = case["tokens"], case["n"], case["k"], case["group"]
    w = (_unpacked(s["w"]).view(N, K // G, G) * s["w_scale"].float()[:, :, None]).view(N, K)
    y = torch.matmul(s["x"].float(), w.t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(s["x"].dtype)


def _places(s):
    """Sequence and position of every new token."""
    t = torch.arange(s["T"], device=DEVICE)
    b = torch.searchsorted(s["starts"][1:].long(), t, right=True)
    return b, s["lens"][b].long() - s["starts"][b + 1].long() + t


def _turn(x, c, n, style, rot):
    x = x.float()
    head, rest = x[..., :rot], x[..., rot:]
    if style == "half":
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        head = torch.cat((a * c - b * n, b * c + a * n), dim=-1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack((a * c - b * n, b * c + a * n), dim=-1).flatten(-2)
    return torch.cat((head, rest), dim=-1)


def _append_plain(s, q, k, v):
    case, rot = s["case"], s["case"]["rot"]
    b, p = _places(s)
    cs = s["cos_sin"][p]
    c, n = cs[:, None, :rot // 2], cs[:, None, rot // 2:]
    page, row = s["table"][b, p // case["page"]].long(), p % case["page"]
    for which, x in (("k", _turn(k, c, n, case["style"], rot)), ("v", v.float())):
        f = s[which + "_scale"].to(torch.bfloat16).float()
        s[which][page, row] = _packed(torch.clamp(torch.round(x * (1 / f)), -8, 7).to(torch.int8))
    return _turn(q, c, n, case["style"], rot).to(q.dtype)


def _attend_plain(s):
    case = s["case"]
    P, D, H, K = case["page"], case["dim"], case["heads"], case["kv_heads"]
    B, L, M, G = case["batch"], s["longest"], s["most"], case["heads"] // case["kv_heads"]
    lens, new = s["lens"].long(), (s["starts"][1:] - s["starts"][:-1]).long()
    j = torch.arange(L, device=DEVICE)
    page, row = s["table"][:, j // P].long(), (j % P).expand(B, L)
    there = j < lens[:, None]
    k, v = (_unpacked(s[n][page, row]).mul_(s[n + "_scale"].to(torch.bfloat16).float()).masked_fill_(~there[:, :, None, None], 0.0)
            .transpose(1, 2) for n in ("k", "v"))                                                        # [B, K, L, D]
    i = torch.arange(M, device=DEVICE)
    at = (s["starts"][:-1].long()[:, None] + i).clamp_(max=s["T"] - 1)
    q = s["q"][at].float().view(B, M, K, G, D).permute(0, 2, 3, 1, 4).reshape(B, K, G * M, D)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(D ** -0.5).view(B, K, G, M, L)
    seen = there[:, None, :].expand(B, M, L)
    if case["causal"]:
        seen = seen & (j <= (lens - new)[:, None, None] + i[:, None])
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    x.sub_(top).exp_()
    total = x.sum(dim=-1, keepdim=True)
    o = torch.matmul(x.view(B, K, G * M, L), v).view(B, K, G, M, D) / total.clamp(min=1e-38)
    lse = (top + total.log()).squeeze(-1)
    b, _ = _places(s)
    m = torch.arange(s["T"], device=DEVICE) - s["starts"][b].long()
    o = o.permute(0, 3, 1, 2, 4)[b, m].reshape(s["T"], H, D).to(s["q"].dtype)
    return {"out": o, "lse": lse.permute(0, 3, 1, 2)[b, m].reshape(s["T"], H)}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _held(s, which):
    """What the cache holds, in 64 bits: the low code of a byte, sign-extended by a multiplication, then the high one."""
    b = s[which].to(torch.int32)
    signed = torch.stack(((b << 28) >> 28, (b << 24) >> 28), dim=-1).flatten(-2)
    return signed.double() * s[which + "_scale"].to(torch.bfloat16).double()


def _fl32(x):
    return x.float().double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        N, K, G = case["n"], case["k"], case["group"]
        y = torch.zeros((case["tokens"], N), dtype=torch.float64, device=DEVICE)
        for g in range(K // G):                       # group by group, as the definition sums
            b = s["w"][:, g * G // 2:(g + 1) * G // 2].to(torch.int32)
            x = s["x"][:, g * G:(g + 1) * G].double()
            part = x[:, 0::2] @ ((b << 28) >> 28).double().T + x[:, 1::2] @ ((b << 24) >> 28).double().T
            y += part * s["w_scale"][:, g].double()
        return y if s["bias"] is None else y + s["bias"].double()
    lens, new = _lengths(case)
    P, D, H, K = case["page"], case["dim"], case["heads"], case["kv_heads"]
    table = s["table"].cpu()
    first = 0
    if case["op"] == "append":
        rot = case["rot"]
        stands = [_held(s, "k"), _held(s, "v")]
        q_out = torch.empty((s["T"], H, D), dtype=torch.float64, device=DEVICE)
        left = torch.arange(rot // 2, device=DEVICE) if case["style"] == "half" else torch.arange(0, rot, 2, device=DEVICE)
        right = left + (rot // 2 if case["style"] == "half" else 1)
        for b, (l, m) in enumerate(zip(lens, new)):
            x = s["qkv"][first:first + m].double()
            co, si = (s["cos_sin"][l - m:l, None, i:i + rot // 2].double() for i in (0, rot // 2))
            # a pair of q's coordinates is a complex number, turned by multiplying it with cos + i sin
            z = torch.complex(x[:, :H, left], x[:, :H, right]) * torch.complex(co, si)
            q_out[first:first + m] = x[:, :H]
            q_out[first:first + m, :, left], q_out[first:first + m, :, right] = z.real, z.imag
            # A code is defined by its fp32 operations, each rounded once: the nearest code of another arithmetic can be the
            # next one.  In 64 bits each result is exact, or so close that rounding it to fp32 is the operation's one rounding.
            kx, kl, kr = x[:, H:H + K].clone(), x[:, H:H + K, left], x[:, H:H + K, right]
            kx[..., left] = _fl32(_fl32(kl * co) - _fl32(kr * si))
            kx[..., right] = _fl32(_fl32(kr * co) + _fl32(kl * si))
            pos = torch.arange(l - m, l)
            page, row = table[b, pos // P].long().to(DEVICE), (pos % P).to(DEVICE)
            for which, y in enumerate((kx, x[:, H + K:])):
                f = (s["k_scale"], s["v_scale"])[which].to(torch.bfloat16).double()
                stands[which][page, row] = _fl32(y * _fl32(1 / f)).round().clamp(-8, 7) * f
            first += m
        return {"q": q_out, "kv": torch.stack(stands)}
    out = torch.zeros((s["T"], H, D), dtype=torch.float64, device=DEVICE)
    lse = torch.full((s["T"], H), -math.inf, dtype=torch.float64, device=DEVICE)
    held = {n: s[n] for n in ("k", "v")}
    for b, (l, m) in enumerate(zip(lens, new)):
        pages = table[b, :-(-l // P)].long().to(DEVICE)
        mine = {n: _held({n: held[n][pages], n + "_scale": s[n + "_scale"]}, n).transpose(1, 2) for n in held}
        for h in range(K):
            kh, vh = (mine[n][:, h].reshape(-1, D)[:l] for n in ("k", "v"))
            for c in range(h * (H // K), (h + 1) * (H // K)):
                logits = s["q"][first:first + m, c].double() @ kh.T / math.sqrt(D)
                if case["causal"]:
                    logits += torch.full((m, l), -math.inf, dtype=torch.float64, device=DEVICE).triu_(l - m + 1)
                lse[first:first + m, c] = torch.logsumexp(logits, dim=1)
                out[first:first + m, c] = torch.softmax(logits, dim=1) @ vh
        first += m
    return {"out": out, "lse": lse}
