"""The few-token linear with 4-bit weights and group factors, and the quantizer that makes its weights."""
import numpy as np
import pytest
import torch

import kv4_reference as R4
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # half an ulp, relative


def problem(T, N, K, group, dtype, bias=False, seed=0):
    g = torch.Generator().manual_seed(seed + 7 * T + N + K)
    x = torch.randn((T, K), generator=g).to(dtype)
    codes = torch.randint(-8, 8, (N, K), generator=g, dtype=torch.int8)
    scale = ((torch.rand((N, K // group), generator=g) + 0.1) * 0.02).to(dtype)
    b = torch.randn((N,), generator=g).to(dtype) if bias else None
    return x, codes, scale, b


def exact(x, codes, scale, bias):
    """y in 64 bits and how far off the kernel may be.  More than 2 tokens: products are exact, and a sum of K of them, taken by
    groups and then over the groups, with K + K / group + 32 additions at most, is off by 2^-23 (the tensor cores may truncate) of
    the sum of the magnitudes each.  Up to 2 tokens: an x is off by at most 2^-22 of the largest of its 256 columns, a group's
    sum is exact, and over the groups there are at most K / group + 40 roundings of 2^-24; the three digits' magnitudes add up to
    at most twice the value's (and 2^-13 of the largest for a value that has fewer).  One narrowing, which may also underflow."""
    N, K = codes.shape
    group = K // scale.shape[1]
    w = (codes.double().view(N, -1, group) * scale.double()[:, :, None]).view(N, K)
    y, size = x.double() @ w.T, x.double().abs() @ w.abs().T
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    if x.shape[0] > 2:
        inner = (K + K // group + 32) * 2.0 ** -23 * size
    else:
        most = torch.nn.functional.pad(x.double().abs(), (0, -K % 256)).view(x.shape[0], -1, 256).amax(dim=2)
        reach = most.repeat_interleave(256, dim=1)[:, :K] @ w.abs().T
        inner = 2.0 ** -22 * reach + (K // group + 40) * 2.0 ** -24 * (2 * size + 2.0 ** -13 * reach)
    tol = UNIT[x.dtype] * y.abs() + inner * (1 + UNIT[x.dtype]) + 2.0 ** -25
    return y.numpy(), tol.numpy()


def run(x, codes, scale, bias, stream=None):
    y = torch.full((x.shape[0], codes.shape[0]), 7.0, dtype=x.dtype, device="cuda")
    on = [t if t is None else t.cuda() for t in (x, R4.packed(codes), scale, bias)]
    P.sasq_w4_linear(on[0], on[1], on[2], y, bias=on[3], stream=stream)
    assert P.sasq_device_status() == 0
    return y.cpu()


def check(*case, **kw):
    data = problem(*case, **kw)
    y = run(*data)
    want, tol = exact(*data)
    assert (np.abs(y.double().numpy() - want) <= tol).all()
    return y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 64, 65, 100])
def test_tokens(T, group, dtype):
    check(T, 200, 1024, group, dtype, bias=T % 2 == 0)


@pytest.mark.parametrize("T", [1, 5, 12, 40])
@pytest.mark.parametrize("N", [1, 7, 15, 16, 17, 31, 33, 63, 65, 127, 129, 1000, 5003])
def test_rows(N, T):
    check(T, N, 512, 128, torch.bfloat16, bias=N % 2 == 1)


@pytest.mark.parametrize("T", [1, 3, 16, 33])
@pytest.mark.parametrize("K,group", [(32, 32), (64, 32), (64, 64), (96, 32), (128, 128), (160, 32), (192, 64), (256, 128), (1120, 32),
                                     (1216, 64), (1152, 128), (4096 + 32, 32), (8192 + 64, 64), (13824, 128), (16384, 128)])
def test_columns(K, group, T):
    check(T, 136, K, group, torch.float16)


@pytest.mark.parametrize("T,N,K", [(1, 4096, 4096), (7, 22016, 512), (1, 30000, 256), (16, 11008, 1024), (61, 6144, 1024), (2, 40, 32768)])
def test_sizes_of_layers(T, N, K):
    """More row tiles than the device holds at once, and few with long columns (clusters)."""
    check(T, N, K, 128, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_code_factor_and_column(dtype):
    """Integers: every partial sum is exact, so every bit of y is."""
    T, N, K = 9, 48, 512
    for group in (32, 64, 128):
        g = torch.Generator().manual_seed(group)
        codes = (torch.arange(N)[:, None] * 5 + torch.arange(K)[None] * 3) % 16 - 8
        scale = 2.0 ** torch.randint(-2, 3, (N, K // group), generator=g).double()
        x = torch.zeros((T, K), dtype=dtype)
        for t in range(T):
            at = torch.randperm(K, generator=g)[:12]
            x[t, at] = torch.randint(1, 5, (12,), generator=g).to(dtype)
        y = run(x, codes.to(torch.int8), scale.to(dtype), None)
        w = (codes.double().view(N, -1, group) * scale[:, :, None]).view(N, K)
        assert torch.equal(y.double(), (x.double() @ w.T).to(dtype).double())


@pytest.mark.parametrize("dtype,by", [(torch.bfloat16, 2.0 ** 60), (torch.bfloat16, 2.0 ** -60), (torch.float16, 2.0 ** -14)])
def test_numbers_at_the_ends_of_their_types(dtype, by):
    x, codes, scale, _ = problem(5, 64, 256, 64, dtype)
    x = (x.double() * by).to(dtype)                        # fp16: subnormal numbers
    y = run(x, codes, scale, None)
    want, tol = exact(x, codes, scale, None)
    tol = tol - 2.0 ** -25 + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)
    assert (np.abs(y.double().numpy() - want) <= tol).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("T", [6, 20])
def test_a_token_that_is_not_finite_reaches_no_other(T, bad):
    x, codes, scale, _ = problem(T, 80, 256, 128, torch.bfloat16)
    want = run(x, codes, scale, None)
    x[3, 17] = bad
    y = run(x, codes, scale, None)
    others = [t for t in range(T) if t != 3]
    assert torch.equal(y[others], want[others]) and not torch.isfinite(y[3][codes[:, 17] != 0]).any()


def test_no_tokens_streams_and_replays():
    x, codes, scale, _ = problem(4, 96, 512, 128, torch.bfloat16)
    empty = torch.empty((0, 512), dtype=torch.bfloat16, device="cuda")
    w, s = R4.packed(codes).cuda(), scale.cuda()
    P.sasq_w4_linear(empty, w, s, torch.empty((0, 96), dtype=torch.bfloat16, device="cuda"))
    want = run(x, codes, scale, None)
    side = torch.cuda.Stream()
    xd, y = x.cuda(), torch.zeros((4, 96), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    P.sasq_w4_linear(xd, w, s, y, stream=side)
    side.synchronize()
    assert torch.equal(y.cpu(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.sasq_w4_linear(xd, w, s, y)
    x2 = problem(4, 96, 512, 128, torch.bfloat16, seed=3)[0]
    xd.copy_(x2)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y.cpu(), run(x2, codes, scale, None))


def test_a_chain_of_linears():
    """Each reads what the one before it writes, while it may already be fetching its weights."""
    n, links = 512, 6
    x = torch.randn((3, n), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    chain = [problem(1, n, n, 64, torch.bfloat16, seed=i)[1:3] for i in range(links)]
    ys = [torch.zeros((3, n), dtype=torch.bfloat16, device="cuda") for _ in range(links)]
    on = [(R4.packed(c).cuda(), s.cuda()) for c, s in chain]
    xd = x.cuda()
    for _ in range(3):
        for i in range(links):
            P.sasq_w4_linear(xd if i == 0 else ys[i - 1], *on[i], ys[i])
    torch.cuda.synchronize()
    for i, (c, s) in enumerate(chain):
        want, tol = exact(x if i == 0 else ys[i - 1].cpu(), c, s, None)
        assert (np.abs(ys[i].cpu().double().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,K,group", [(1, 32, 32), (37, 96, 32), (5, 192, 64), (64, 1152, 128), (3001, 256, 128)])
def test_quantizer(N, K, group, dtype):
    """Bit for bit the definition in fp32."""
    w = torch.randn((N, K), generator=torch.Generator().manual_seed(N)) * 0.02
    w[0, :32] = 0.0
    if group == 32:
        w[0, 0] = 0.0
    w[-1, -1] = 3.0
    codes, scale = torch.empty((N, K // 2), dtype=torch.uint8, device="cuda"), torch.empty((N, K // group), dtype=dtype, device="cuda")
    P.sasq_quantize_weight_w4(w.cuda(), codes, scale)
    groups = w.view(N, -1, group)
    s = (groups.abs().amax(dim=2) / 7).to(dtype)
    s = torch.where(s == 0, torch.ones_like(s), s)
    assert torch.equal(scale.cpu(), s)
    want = torch.clamp(torch.round(groups * (1 / s.float())[:, :, None]), -8, 7).to(torch.int8).view(N, K)
    assert torch.equal(codes.cpu(), R4.packed(want))


def test_quantizer_at_the_ends():
    w = torch.zeros((4, 64))
    w[0], w[1], w[2], w[3] = 1e-42, 1e6, 2e38, 0.5
    for dtype, most in ((torch.float16, 65504.0), (torch.bfloat16, 3e38)):
        codes, scale = torch.empty((4, 32), dtype=torch.uint8, device="cuda"), torch.empty((4, 1), dtype=dtype, device="cuda")
        P.sasq_quantize_weight_w4(w.cuda(), codes, scale)
        s = scale.float().cpu()
        assert s[0] == 1.0 and torch.isfinite(s).all() and (s <= most).all() and (s > 0).all()
        got = R4.unpacked(codes.cpu())
        assert (got[0] == 0).all() and (got[1] == 7).all() and (got[2] == 7).all() and (got[3] == 7).all()
