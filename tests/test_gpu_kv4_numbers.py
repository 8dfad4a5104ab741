"""The 4-bit cache's arithmetic: value factors up to fp32's end, and long keys against bounds that count what the kernels add."""
import numpy as np
import pytest
import torch

import kv4_reference as R4
import paper_2512_14481_b200 as P
from test_gpu_kv4_attention import attend, check

pytestmark = pytest.mark.gpu

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # half an ulp, relative


@pytest.mark.parametrize("lens,new,dim", [
    ([150, 1, 90], 1, 64),          # one cluster an item
    ([150, 1, 90], 50, 64),         # many rows, whole items
    ([9000, 40], 1, 128),           # few rows, items cut among blocks
    ([9000, 400], 4, 64),           # the same, 16 rows
    ([9000, 400], 60, 128)])        # many rows, items cut among blocks
@pytest.mark.parametrize("by", [2.0 ** 122, -2.0 ** 122, 2.0 ** -100])
def test_value_factors_to_the_end(lens, new, dim, by):
    """A result is an average of codes times a factor: a number wherever the factor is one."""
    bt = R4.Batch(lens, [min(new, l) for l in lens], 4, 2, dim, 16, torch.bfloat16, seed=4)
    bt.v_scale = bt.v_scale * by
    out, _ = check(bt)
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("steps", [1, 4])
@pytest.mark.parametrize("new,count,hi,dim", [(1, 2, 14000, 128), (1, 30, 6000, 64), (4, 3, 14000, 64), (40, 2, 14000, 128), (1, 5, 900, 128)])
def test_flat_and_stepped_probabilities_over_long_keys(new, count, hi, dim, steps, dtype):
    """Probabilities are powers of two, up to 2^3 apart, so that they are f16 numbers and every partial sum of them times codes
    is an integer below 2^24 of some power of two: exact.  What is left: the exponentials' and the sums' 2^-18 of the sum of the
    magnitudes, as for the other caches, and the narrowing."""
    lens = [hi - 97 * i for i in range(count)]
    bt = R4.Batch(lens, [new] * count, 8, 2, dim, 32, dtype, seed=new + count)
    bt.k_scale = torch.ones_like(bt.k_scale)
    k = bt.k_host.clone()
    k[..., 0] = k[..., 0] & (steps - 1)
    bt.set_codes(k, bt.v_host)
    q = torch.zeros_like(bt.q_wide)
    q[..., 0] = 1
    bt.q_wide, bt.q = q, q.cuda()
    out, lse = attend(bt, causal=False, scale=float(np.log(2)))
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, l in enumerate(lens):
        rows = slice(int(bt.starts[b]), int(bt.starts[b]) + new)
        kh, vh = bt.keys(b)
        for c in range(8):
            p = np.exp2(kh[:, c // 4, 0])
            p_sum = p.sum()
            want, size = p @ vh[:, c // 4] / p_sum, p @ np.abs(vh[:, c // 4]) / p_sum
            assert (np.abs(got[rows, c] - want) <= UNIT[dtype] * np.abs(want) + 2.0 ** -18 * size + 2.0 ** -25).all()
            assert (np.abs(got_lse[rows, c] - np.log(p_sum)) <= 2.0 ** -18 + 2.0 ** -22 * np.log(p_sum)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("new,hi,dim", [(1, 14000, 128), (4, 14000, 64), (40, 9000, 64)])
def test_long_keys_with_faint_logits(new, hi, dim, dtype):
    """Logits of a few tenths: nearly flat probabilities, results that are averages of thousands of codes.

    Of a probability p the second product takes f16(p), off by 2^-11 p, or by 2^-25 of a reference that is 2^7 below the row's
    maximum or lower still.  Few rows: four warps at least share the keys, and their sums of p (c + 8) and of 8 p are off by
    2^-23 of themselves for each of a warp's additions (the tensor cores may truncate).  Many rows: sums of p c over all keys."""
    lens = [hi, hi // 3]
    bt = R4.Batch(lens, [new, new], 8, 2, dim, 64, dtype, seed=new)
    bt.q_wide = (bt.q_wide.float() * 0.02).to(dtype)
    bt.q = bt.q_wide.cuda()
    scale = dim ** -0.5
    out, _ = attend(bt, causal=False, scale=scale)
    got = out.double().cpu().numpy()
    q = bt.q_wide.double().numpy()
    for b, l in enumerate(lens):
        rows = slice(int(bt.starts[b]), int(bt.starts[b]) + new)
        kh, vh = bt.keys(b)
        for c in range(8):
            s = q[rows, c] @ kh[:, c // 4].T * scale
            p = np.exp(s - s.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            f = R4.used(bt.v_scale[c // 4]).double().numpy()
            want, size = p @ vh[:, c // 4], p @ np.abs(vh[:, c // 4])
            qs = np.abs(q[rows, c]) * R4.used(bt.k_scale[c // 4]).double().numpy()
            e = np.maximum(8 * dim * 2.0 ** -22 * qs.max(axis=1) + 2.0 ** -17 * qs.sum(axis=1),
                           (dim + 8) * 2.0 ** -20 * qs.sum(axis=1))[:, None] * scale
            tol = UNIT[dtype] * np.abs(want) + size * (2 * e + 2.0 ** -11 + 2.0 ** -18) + l * 2.0 ** -32 * np.abs(vh).max() + 2.0 ** -25
            if new * 4 <= 16:
                tol = tol + (l / 4 + 40) * 2.0 ** -23 * (want + 16 * f)
            else:
                tol = tol + (l + 40) * 2.0 ** -23 * size
            assert (np.abs(got[rows, c] - want) <= tol).all()


@pytest.mark.parametrize("new", [1, 4, 50])
@pytest.mark.parametrize("q_by,f_by,s_by", [(60, -60, 0), (-60, 60, 0), (-90, 60, 30), (-80, 112, -32), (118, -100, -18), (122, -92, -30), (110, -116, 6)])
def test_powers_of_two_cancel(new, q_by, f_by, s_by):
    """Queries, key factors and the scale times powers of two whose product is 1: the same logits, bit for bit."""
    results = []
    for by in ((0, 0, 0), (q_by, f_by, s_by)):
        bt = R4.Batch([400, 333], [new, new], 4, 2, 128, 16, torch.bfloat16, seed=4)
        bt.k_scale = bt.k_scale * 2.0 ** by[1]
        bt.q_wide = bt.q_wide * 2.0 ** by[0]
        bt.q = bt.q_wide.cuda()
        results.append(attend(bt, scale=0.0877 * 2.0 ** by[2]))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])


@pytest.mark.parametrize("lens,new,dim", [([1, 40], [2, 2], 128), ([2, 9000], [4, 4], 64), ([3, 9000], [40, 60], 128), ([10, 5], [90, 90], 64)])
def test_rows_without_keys_are_plus_zero_under_negative_factors(lens, new, dim):
    bt = R4.Batch(lens, new, 4, 2, dim, 16, torch.bfloat16, seed=3)
    bt.v_scale = -bt.v_scale
    out, lse = check(bt)
    empty = torch.isneginf(lse)
    assert empty.any() and (out[empty].view(torch.int16) == 0).all()
