"""The 4-bit linear at the ends of its numbers, for each of its three ways (one or two tokens, up to 16, more): far tokens and
factors, tokens that are not finite, and one loud element among faint ones."""
import numpy as np
import pytest
import torch

import paper_2512_14481_b200 as P
from test_gpu_w4_linear import exact, problem, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 2, 5, 20])
@pytest.mark.parametrize("dtype,x_by,s_by", [
    (torch.bfloat16, 2.0 ** 60, 1.0), (torch.bfloat16, 2.0 ** -60, 1.0), (torch.float16, 2.0 ** -14, 1.0), (torch.bfloat16, 2.0 ** 110, 2.0 ** -60),
    (torch.bfloat16, 2.0 ** -50, 2.0 ** 130), (torch.bfloat16, 2.0 ** -80, 2.0 ** 120), (torch.bfloat16, 2.0 ** 100, 2.0 ** -110),
    (torch.bfloat16, 2.0 ** -90, 2.0 ** 60)])
def test_numbers_at_the_ends_of_their_types(T, dtype, x_by, s_by):
    """Factors of `problem` lie between 2^-9 and 2^-5.  Sums of a group and of all groups are fp32 numbers throughout."""
    x, codes, scale, _ = problem(T, 64, 512, 64, dtype)
    x, scale = (x.double() * x_by).to(dtype), (scale.double() * s_by).to(dtype)
    y = run(x, codes, scale, None)
    want, tol = exact(x, codes, scale, None)
    tol = tol - 2.0 ** -25 + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)
    assert (np.abs(y.double().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("T,t", [(1, 0), (2, 0), (2, 1)])
def test_one_or_two_tokens_of_which_one_is_not_finite(T, t, bad, dtype):
    """All of that token's row is not finite, whatever the codes; the other token's is as it was."""
    x, codes, scale, _ = problem(T, 80, 1024, 128, dtype)
    codes[::2, 700] = 0
    want = run(x, codes, scale, None)
    x[t, 700] = bad
    y = run(x, codes, scale, None)
    assert not torch.isfinite(y[t]).any()
    assert T == 1 or torch.equal(y[1 - t], want[1 - t])


@pytest.mark.parametrize("by", [2.0 ** 10, 2.0 ** 15])
@pytest.mark.parametrize("T", [1, 2, 4])
def test_a_loud_element_among_faint_ones(T, by):
    """Rows whose code in the loud column is 0 are sums of the faint ones alone."""
    x, codes, scale, _ = problem(T, 64, 512, 64, torch.bfloat16)
    x[:, 300] = torch.tensor([by * (1.25 if t % 2 else -1.0) for t in range(T)]).to(x.dtype)
    codes[::2, 300] = 0
    y = run(x, codes, scale, None)
    want, tol = exact(x, codes, scale, None)
    assert (np.abs(y.double().numpy() - want) <= tol).all()
    assert (np.abs(want[:, ::2]).max() < by / 8)


@pytest.mark.parametrize("T", [1, 2, 5, 20])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_factor_that_is_not_finite_reaches_no_other_column(T, bad):
    x, codes, scale, _ = problem(T, 80, 576, 64, torch.bfloat16)
    want = run(x, codes, scale, None)
    scale[33, 8] = bad
    scale[79, 2] = bad
    y = run(x, codes, scale, None)
    others = [n for n in range(80) if n not in (33, 79)]
    assert torch.equal(y[:, others], want[:, others]) and not torch.isfinite(y[:, [33, 79]]).any()


@pytest.mark.parametrize("T", [1, 2, 3, 9, 17, 33, 70])
@pytest.mark.parametrize("N,K,group", [(200, 1056, 32), (1000, 4160, 64), (130, 13824, 128)])
def test_what_ran_before_does_not_show(N, K, group, T):
    """The same call behind linears of every kind that leave loud numbers, or zeros, in shared memory."""
    x, codes, scale, bias = problem(T, N, K, group, torch.float16, bias=True)
    w = torch.randint(0, 256, (19000, 1024), dtype=torch.uint8, device="cuda")
    w_scale = torch.rand((19000, 32), device="cuda").to(torch.float16)
    results = []
    for loud in (1000.0, 0.0):
        for tokens in (2, 8, 16, 32, 64):
            before = (torch.randn((tokens, 2048), device="cuda") * loud).to(torch.float16)
            P.sasq_w4_linear(before, w, w_scale, torch.empty((tokens, 19000), dtype=torch.float16, device="cuda"))
        results.append(run(x, codes, scale, bias))
    assert torch.equal(results[0], results[1])
