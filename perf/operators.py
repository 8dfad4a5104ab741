"""The paged-cache operators as they are used in serving: what is run, on which sizes, and what each pass has to move.

Two operators: `append` (rotary positions on q and k, k and v appended to a paged cache) and `attend` (attention of the
new tokens of a batch of sequences over that cache).  Each has a plain form in elementary torch operations on fp32
values, and the framework's own calls (where `own` is true)."""
import math
import random

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------------
def _case(op, name=None, dt="bf16", kv="16", heads=32, kv_heads=32, dim=128, page=16, batch=1, ctx=(0, 0), new=(1, 1),
          causal=True, layout="heads", style="half", rot=None):
    """ctx: tokens that the cache holds before the new ones, from the shortest to the longest sequence; new: new tokens."""
    c = {"op": op, "dt": dt, "kv": kv, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "batch": batch,
         "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": new[0], "new_hi": new[1], "layout": layout}
    if op == "append":
        c["style"] = style
        c["rot"] = dim if rot is None else rot
    else:
        c["causal"] = causal
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's next token in a LLaMA-2-7B-shaped layer: all latency
        _case("append", "append one token", ctx=(1000, 1000)),
        # a decode step of a full batch with grouped heads, ragged contexts
        _case("append", "append decode 128", heads=32, kv_heads=8, batch=128, ctx=(17, 6000), page=32),
        # whole prompts of a LLaMA-2-13B-shaped layer (40 heads), a stretch of tokens from an odd place on
        _case("append", "append prompt fp16", dt="fp16", heads=40, kv_heads=40, batch=3, ctx=(0, 77), new=(1111, 4099)),
        # chunked prefill into the int8 cache, interleaved pairs, tokens-first pages
        _case("append", "append chunk int8", kv="int8", heads=32, kv_heads=8, batch=8, ctx=(5, 3001), new=(512, 512),
              page=64, layout="tokens", style="pairs"),
        # one user's next token, LLaMA-2-7B-shaped, about a thousand tokens in
        _case("attend", "decode one", ctx=(1000, 1000)),
        # a decode step of a batch of ragged conversations, grouped heads
        _case("attend", "decode 64 ragged", heads=32, kv_heads=8, batch=64, ctx=(30, 4500), page=32),
        # long documents in the int8 cache, a few readers
        _case("attend", "decode long int8", kv="int8", heads=32, kv_heads=8, batch=8, ctx=(8000, 32000), page=64),
        # a draft's seven tokens checked at once, heads of 64, fp16, odd group of five
        _case("attend", "verify 7 fp16", dt="fp16", heads=40, kv_heads=8, dim=64, batch=16, ctx=(100, 3000), new=(7, 7),
              layout="tokens"),
        # decode and chunked prefill in one batch, 13B-shaped heads
        _case("attend", "mixed batch", heads=40, kv_heads=40, batch=12, ctx=(1, 2500), new=(1, 300)),
        # a chunk of a long prompt over the int8 cache
        _case("attend", "chunk 1024 int8", kv="int8", heads=32, kv_heads=8, ctx=(15000, 15000), new=(1024, 1024), page=128),
        # a whole prompt of a LLaMA-2-7B-shaped layer at once: the largest
        _case("attend", "prompt 8192", new=(8192, 8192), page=64),
        # all queries see all keys (an encoder's states in the cache), ragged
        _case("attend", "every key fp16", dt="fp16", heads=16, kv_heads=4, batch=4, ctx=(0, 900), new=(333, 1500), causal=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("append", "attend", "attend"))
        group = rng.choice((1, 1, 2, 3, 4, 5, 7, 8))
        kv_heads = rng.choice((1, 2, 4, 5, 8, 8, 16, 32, 40))
        dim = rng.choice((64, 128, 128))
        kind = rng.choice(("decode", "few", "chunk", "prompt"))
        batch = _log(rng, 1, 128) if kind == "decode" else _log(rng, 1, 32) if kind == "few" else _log(rng, 1, 12)
        hi = _log(rng, 1, 32000) if kind != "prompt" else _log(rng, 1, 200)
        new_hi = 1 if kind == "decode" else rng.randint(2, 16) if kind == "few" else _log(rng, 17, 1500) if kind == "chunk" \
            else _log(rng, 100, 8192)
        new_lo = 1 if kind == "decode" else rng.randint(1, new_hi)
        c = _case(op, dt=rng.choice(("bf16", "bf16", "fp16")), kv=rng.choice(("16", "16", "int8")), heads=group * kv_heads,
                  kv_heads=kv_heads, dim=dim, page=rng.choice((16, 32, 64, 128)), batch=batch, ctx=(rng.randint(0, hi), hi),
                  new=(new_lo, new_hi), causal=rng.random() < 0.85, layout=rng.choice(("heads", "tokens")),
                  style=rng.choice(("half", "half", "pairs")), rot=rng.choice((dim, dim, dim // 2)))
        if c["heads"] > 64:
            continue
        lens, new_ = _lengths(c)
        w, longest, most = work(c), max(lens), max(new_)
        if op == "append" and w["bytes"] <= 3.4e8 and sum(lens) * kv_heads * dim <= 1 << 28:
            return c
        if op == "attend" and w["flops"] <= 5.5e11 and w["bytes"] <= 1.2e9 and batch * longest * kv_heads * dim <= 1 << 29 \
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
    lens, new = _lengths(case)
    T, D, H, K = sum(new), case["dim"], case["heads"], case["kv_heads"]
    held = 1 if case["kv"] == "int8" else 2
    if case["op"] == "append":
        places = len({p for l, m in zip(lens, new) for p in range(l - m, l)})
        return {"bytes": T * (H * D * 4 + K * D * 2 * (2 + held)) + places * case["rot"] * 4, "flops": 3 * T * (H + K) * case["rot"]}
    return {"bytes": sum(lens) * K * D * 2 * held + T * H * (D * 4 + 4), "flops": 4 * D * H * _pairs(case)}


# ---------------------------------------------------------------------------------------------------------------------
# the inputs
# ---------------------------------------------------------------------------------------------------------------------
def _values(shape, dt, gen, wide=0.02, by=4.0):
    """Normal values with a few louder channels, as projections of a decoder layer have them."""
    x = torch.randn(shape, generator=gen, device=DEVICE)
    loud = (torch.rand(shape[-2:], generator=gen, device=DEVICE) < wide).float() * (by - 1) + 1
    return x.mul_(loud).to(dt)


def _pages(case, n_pages, gen, quantized):
    """The cache's memory [pages, page, kv heads, dim] in the case's order, with what earlier requests left in it."""
    P, K, D = case["page"], case["kv_heads"], case["dim"]
    x = _values((n_pages, P, K, D), DTYPES[case["dt"]], gen)
    scale = None
    if quantized:
        scale = x.float().abs().amax(dim=(0, 1, 3)) * 0.8 / 127
        x = torch.clamp(torch.round(x.float() / scale[None, None, :, None]), -128, 127).to(torch.int8)
    if case["layout"] == "heads":
        x = x.transpose(1, 2).contiguous().transpose(1, 2)
    return x, scale


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    lens, new = _lengths(case)
    dt, P, D, H, K = DTYPES[case["dt"]], case["page"], case["dim"], case["heads"], case["kv_heads"]
    T, B = sum(new), len(lens)
    need = [-(-l // P) for l in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.zeros((B, max(need)), dtype=torch.int32, device=DEVICE)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    k, k_scale = _pages(case, n_pages, gen, case["kv"] == "int8")
    v, v_scale = _pages(case, n_pages, gen, case["kv"] == "int8")
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    s = {"case": case, "k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale, "table": table,
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
    else:
        s["q"] = (_values((T, H, D), torch.float32, gen) * 1.5).to(dt)
        s["out"] = torch.empty((T, H, D), dtype=dt, device=DEVICE)
        s["lse"] = torch.empty((T, H), dtype=torch.float32, device=DEVICE)
    if own:  # the handles and the scratch memory that a serving loop keeps over its steps
        import paper_2512_14481_b200 as P_
        s["lib"] = P_
        s["cache"] = P_.KVCache(k, v, k_scale, v_scale)
        s["batch"] = P_.PagedBatch(table, s["lens"], s["starts"], T, s["most"], s["longest"])
        if case["op"] == "attend":
            s["ws"] = torch.empty(P_.sasq_paged_attention_workspace(s["cache"], s["batch"], H), dtype=torch.uint8, device=DEVICE)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if case["op"] == "append":
        H, K = case["heads"], case["kv_heads"]
        q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + K], s["qkv"][:, H + K:]
        if own:
            s["lib"].sasq_rope_kv_append(s["cache"], s["batch"], q, k, v, s["q_out"], s["cos_sin"],
                                         interleaved=case["style"] == "pairs")
            q_out = s["q_out"]
        else:
            q_out = _append_plain(s, q, k, v)
        if case["kv"] == "int8":
            return {"q": q_out, "k": s["k"].float() * s["k_scale"][:, None], "v": s["v"].float() * s["v_scale"][:, None]}
        return {"q": q_out, "k": s["k"], "v": s["v"]}
    if own:
        s["lib"].sasq_paged_attention(s["cache"], s["batch"], s["q"], s["out"], s["ws"], lse=s["lse"],
                                      scale=case["dim"] ** -0.5, causal=case["causal"])
        return {"out": s["out"], "lse": s["lse"]}
    return _attend_plain(s)


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
    kr, vr = _turn(k, c, n, case["style"], rot), v.float()
    if case["kv"] == "int8":
        kr = torch.clamp(torch.round(kr * (1 / s["k_scale"])[:, None]), -128, 127)
        vr = torch.clamp(torch.round(vr * (1 / s["v_scale"])[:, None]), -128, 127)
    s["k"][page, row] = kr.to(s["k"].dtype)
    s["v"][page, row] = vr.to(s["v"].dtype)
    return _turn(q, c, n, case["style"], rot).to(q.dtype)


def _attend_plain(s):
    case = s["case"]
    P, D, H, K = case["page"], case["dim"], case["heads"], case["kv_heads"]
    B, L, M, G = case["batch"], s["longest"], s["most"], case["heads"] // case["kv_heads"]
    lens, new = s["lens"].long(), (s["starts"][1:] - s["starts"][:-1]).long()
    j = torch.arange(L, device=DEVICE)
    page, row = s["table"][:, j // P].long(), (j % P).expand(B, L)
    there = j < lens[:, None]
    k = s["k"][page, row].float().masked_fill_(~there[:, :, None, None], 0.0).transpose(1, 2)       # [B, K, L, D]
    v = s["v"][page, row].float().masked_fill_(~there[:, :, None, None], 0.0).transpose(1, 2)
    if case["kv"] == "int8":
        k, v = k * s["k_scale"][:, None, None], v * s["v_scale"][:, None, None]
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
def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _lengths(case)
    P, D, H, K = case["page"], case["dim"], case["heads"], case["kv_heads"]
    table = s["table"].cpu()
    first = 0
    if case["op"] == "append":
        rot = case["rot"]
        stands = [s["k"].double(), s["v"].double()]
        factors = [s["k_scale"], s["v_scale"]]
        if case["kv"] == "int8":
            stands = [x * f.double()[:, None] for x, f in zip(stands, factors)]
        q_out = torch.empty((s["T"], H, D), dtype=torch.float64, device=DEVICE)
        # a pair of coordinates is a complex number, turned by multiplying it with cos + i sin
        left = torch.arange(rot // 2, device=DEVICE) if case["style"] == "half" else torch.arange(0, rot, 2, device=DEVICE)
        right = left + (rot // 2 if case["style"] == "half" else 1)
        for b, (l, m) in enumerate(zip(lens, new)):
            x = s["qkv"][first:first + m].double()
            unit = torch.complex(s["cos_sin"][l - m:l, :rot // 2].double(), s["cos_sin"][l - m:l, rot // 2:].double())
            z = torch.complex(x[:, :H + K, left], x[:, :H + K, right]) * unit[:, None]
            x[:, :H + K, left], x[:, :H + K, right] = z.real, z.imag
            q_out[first:first + m] = x[:, :H]
            pos = torch.arange(l - m, l)
            page, row = table[b, pos // P].long().to(DEVICE), (pos % P).to(DEVICE)
            for which, y in enumerate((x[:, H:H + K], x[:, H + K:])):
                if case["kv"] == "int8":
                    f = factors[which].double()[:, None]
                    y = (y / f).round().clamp(-128, 127) * f
                stands[which][page, row] = y
            first += m
        return {"q": q_out, "k": stands[0], "v": stands[1]}
    out = torch.zeros((s["T"], H, D), dtype=torch.float64, device=DEVICE)
    lse = torch.full((s["T"], H), -math.inf, dtype=torch.float64, device=DEVICE)
    for b, (l, m) in enumerate(zip(lens, new)):
        pages = table[b, :-(-l // P)].long().to(DEVICE)
        for h in range(K):
            kh, vh = (s[n][pages, :, h].reshape(-1, D)[:l].double() for n in ("k", "v"))
            if case["kv"] == "int8":
                kh, vh = kh * s["k_scale"][h].double(), vh * s["v_scale"][h].double()
            for g in range(H // K):
                c = h * (H // K) + g
                logits = s["q"][first:first + m, c].double() @ kh.T / math.sqrt(D)
                if case["causal"]:
                    logits += torch.full((m, l), -math.inf, dtype=torch.float64, device=DEVICE).triu_(l - m + 1)
                lse[first:first + m, c] = torch.logsumexp(logits, dim=1)
                out[first:first + m, c] = torch.softmax(logits, dim=1) @ vh
        first += m
    return {"out": out, "lse": lse}
