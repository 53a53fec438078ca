"""Attention at the edges of its numbers, on the GPU through the C ABI: large scores, values that are not finite, weights near a type's smallest.

u = 2^-24 is half a unit in the last place of 32 bits.
"""
import math

import numpy as np
import pytest
import torch

from oracle import attention as at
from tests.test_gpu_attention import HALF, IDS, TYPES, U, Case, ctx, desc_of, f64, qrm  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

# (queries, keys, query heads, key heads, elements): one tile, many tiles, splits that are joined, few rows, rows of two wavefronts
LARGE = [(1, 1, 1, 1, 64), (40, 3, 2, 2, 64), (3, 5000, 2, 1, 64), (100, 700, 2, 2, 128), (70, 90, 1, 1, 512), (40, 3000, 1, 1, 512), (1, 900, 4, 1, 512)]


@pytest.mark.parametrize("power", [-3, 4, 37, 80])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("shape", LARGE, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_large_scores(ctx, qrm, dtype, shape, sign, power):
    """Scores of 1e8 and more, up to 1e33: three keys (first, middle and last) have the largest, all others half of it or twice (where negative).  Each of the three has
    a third of the weight: differences of 0 are exact in any format, those of the others leave nothing.  o: a few roundings of the mean and half a step of the type; lse: the
    sums of powers of two are exact, so the product with the scale and the sum with log 3 are all that is rounded."""
    lq, lk, heads, kv, d = shape
    top = 1.25 * 2.0 ** (11 if dtype == torch.float16 or power < 80 else 20)
    scale = 2.0 ** min(power, 60)
    g = torch.Generator().manual_seed(lk + d)
    winners = sorted({0, lk // 2, lk - 1})
    q = torch.full((2, lq, heads, d), sign * top, dtype=dtype, device="cuda")
    k = torch.full((2, lk, kv, d), top / 2 if sign > 0 else top, dtype=dtype, device="cuda")
    k[:, winners] = top if sign > 0 else top / 2
    v = (torch.randn((2, lk, kv, d), generator=g) + 0.5).to(dtype).cuda()
    o, lse = torch.empty_like(q), torch.empty((2, heads, lq), device="cuda")
    ctx.qrm_attention(desc_of(qrm, q, k, v, o, False, scale), q, k, v, o, lse, None, None, 0)
    mean = f64(v)[:, winners].mean(axis=1)                                     # [2, kv, d]
    want = np.repeat(mean, heads // kv, axis=1)[:, None]
    size = np.repeat(np.abs(f64(v)[:, winners]).mean(axis=1), heads // kv, axis=1)[:, None]
    assert (np.abs(f64(o) - want) <= 8 * U * size + HALF[dtype] * np.abs(want) * 1.01).all()
    want_lse = scale * sign * d * top * (top if sign > 0 else top / 2) + math.log(len(winners))
    assert float((lse.double() - want_lse).abs().max()) <= 4 * U * abs(want_lse)


@pytest.mark.parametrize("shape", [(3, 5000, 2, 1, 64), (100, 130, 2, 2, 64), (70, 90, 1, 1, 512), (40, 3000, 1, 1, 512)], ids=str)
@pytest.mark.parametrize("powers", [(40, 30, 60), (100, 100, 0)], ids=["scaled", "raw"])
@pytest.mark.parametrize("dtype", TYPES[:2], ids=IDS[:2])
def test_scores_below_32_bits_are_no_rows_that_see_nothing(ctx, qrm, dtype, powers, shape):
    """Scores of -2^136 after the scale, or -2^206 before it: no numbers, whatever the rows beside them see."""
    lq, lk, heads, kv, d = shape
    q = torch.full((2, lq, heads, d), -2.0 ** powers[0], dtype=dtype, device="cuda")
    k, v = torch.full((2, lk, kv, d), 2.0 ** powers[1], dtype=dtype, device="cuda"), torch.ones((2, lk, kv, d), dtype=dtype, device="cuda")
    q[1, -1] = 0.0                                                             # (scores of zero: the mean of the values)
    o, lse = torch.empty_like(q), torch.empty((2, heads, lq), device="cuda")
    desc = desc_of(qrm, q, k, v, o, False, 2.0 ** powers[2])
    ctx.qrm_attention(desc, q, k, v, o, lse, None, None, 0)
    torch.cuda.synchronize()
    assert bool(torch.isnan(o[0]).all()) and bool(torch.isnan(lse[0]).all()) and bool(torch.isnan(o[1, :-1]).all()) and bool(torch.isnan(lse[1, :, :-1]).all())
    # lk equal weights and values of one: a rounding a key in the sums on either side, and half a step
    assert float((o[1, -1].double() - 1.0).abs().max()) <= 2 * lk * U + HALF[dtype]
    assert float((lse[1, :, -1].double() - math.log(lk)).abs().max()) <= (lk + 16) * U * 1.01
    # one key of score 0 among them has all of the weight
    k[:, lk // 2] = 0.0
    v[:, lk // 2] = 3.0
    ctx.qrm_attention(desc, q, k, v, o, lse, None, None, 0)
    torch.cuda.synchronize()
    assert bool((o[0] == 3.0).all()) and bool((lse[0] == 0.0).all())


@pytest.mark.parametrize("shape", [(3, 5000, 2, 1, 64), (100, 130, 2, 2, 64), (40, 3000, 1, 1, 512)], ids=str)
@pytest.mark.parametrize("dtype", TYPES[:2], ids=IDS[:2])
def test_raw_scores_above_32_bits(ctx, qrm, dtype, shape):
    """One key whose products pass 32 bits' largest: the rows that see it are no numbers, the others are as if it were not there."""
    lq, lk, heads, kv, d = shape
    q = torch.full((1, lq, heads, d), 2.0 ** 70, dtype=dtype, device="cuda")
    k, v = torch.zeros((1, lk, kv, d), dtype=dtype, device="cuda"), torch.ones((1, lk, kv, d), dtype=dtype, device="cuda")
    q[:, -1], k[:, lk // 3] = 0.0, 2.0 ** 70
    o, lse = torch.empty_like(q), torch.empty((1, heads, lq), device="cuda")
    ctx.qrm_attention(desc_of(qrm, q, k, v, o, False, 1.0), q, k, v, o, lse, None, None, 0)
    torch.cuda.synchronize()
    assert bool(torch.isnan(o[0, :-1]).all()) and bool(torch.isnan(lse[..., :-1]).all())
    assert float((o[0, -1].double() - 1.0).abs().max()) <= 2 * lk * U + HALF[dtype]


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("shape", [(1, 5, 2, 1, 64), (3, 5000, 2, 1, 64), (40, 3000, 1, 1, 512), (100, 3000, 1, 1, 128)], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_a_value_that_is_not_finite_reaches_rows_in_which_it_has_no_weight(ctx, qrm, dtype, shape, bad):
    """Keys of the second half have scores 200 under those of the first, weights that 32 bits do not hold: 0 times such a value is no number, however the keys are split."""
    lq, lk, heads, kv, d = shape
    q = torch.full((1, lq, heads, d), 1.0, dtype=dtype, device="cuda")
    k, v = torch.zeros((1, lk, kv, d), dtype=dtype, device="cuda"), torch.ones((1, lk, kv, d), dtype=dtype, device="cuda")
    k[:, lk // 2:, :, 0] = -200.0
    v[0, lk - 1, 0, 3] = bad
    o = torch.empty_like(q)
    ctx.qrm_attention(desc_of(qrm, q, k, v, o, False, 1.0), q, k, v, o, None, None, None, 0)
    torch.cuda.synchronize()
    assert not bool(torch.isfinite(o[..., 3]).any())
    o[..., 3] = 1.0
    assert float((o.double() - 1.0).abs().max()) <= 2 * lk * U + HALF[dtype]


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(100, 130, 4, 2, 64), (90, 40, 2, 1, 512), (3, 5000, 2, 1, 64), (300, 2000, 1, 1, 128), (70, 90, 2, 2, 45)], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_rows_that_see_nothing_stay_zeros_beside_values_that_are_not_finite(ctx, qrm, dtype, shape, causal, bad):
    """Keys and values that are there hold NaNs or infinities: rows that are not there, and the first rows of more queries than keys, have nothing of them."""
    lq, lk, heads, kv, d = shape
    q_len, k_len = [2 * lq // 3, lq, 1], [lk, max(1, min(lk, lq) // 2), lk // 2]
    c = Case(qrm, 3, lq, lk, heads, kv, d, dtype, causal=causal, q_len=q_len, k_len=k_len, seed=3)
    for i, m in enumerate(k_len):
        c.v[i, m - 1] = bad
        c.k[i, m // 2] = bad
    c.forward(ctx)
    c.backward(ctx)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(q_len, k_len)):
        first = max(0, a - b) if causal else 0                                 # rows that see nothing
        for rows in (slice(0, first), slice(a, lq)):
            assert bool((c.o[i, rows] == 0).all()) and bool((c.dq[i, rows] == 0).all()) and bool(torch.isneginf(c.lse[i, :, rows]).all())
        assert bool((c.dk[i, b:] == 0).all()) and bool((c.dv[i, b:] == 0).all())
        assert not bool(torch.isfinite(c.o[i, a - 1]).any())                   # (the last one sees all keys)


@pytest.mark.parametrize("score", [-18.0, -24.0, -28.0, -32.0])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_gradients_of_values_of_little_weight(ctx, qrm, dtype, score):
    """Keys of weight exp(-18) .. exp(-32) in each of 2^15 rows, whose gradients are 2^10: exp(-28) is under 2^-40, the sums are not small.  Half a step each for weights and
    results (f16: 2^-25 at least); a rounding of equal summands for every two rows; a score's 32 + 8 roundings."""
    lq, heads, lk, d = 4096, 8, 256, 32
    q = torch.zeros((1, lq, heads, d), dtype=dtype, device="cuda")
    k, v = (torch.zeros((1, lk, 1, d), dtype=dtype, device="cuda") for _ in range(2))
    q[..., 0], k[..., 0] = 4.0, score / 4.0
    k[0, 77] = 0.0
    do = torch.full_like(q, 2.0 ** 10)
    o, lse, dv = torch.empty_like(q), torch.empty((1, heads, lq), device="cuda"), torch.empty_like(v)
    desc = desc_of(qrm, q, k, v, o, False, 1.0)
    ctx.qrm_attention(desc, q, k, v, o, lse, None, None, 0)
    ctx.qrm_attention_backward(desc, q, k, v, o, do, lse, None, None, dv, None, None, 0)
    torch.cuda.synchronize()
    rows, half, p = lq * heads, HALF[dtype], math.exp(score)
    want = torch.full((lk, d), rows * 2.0 ** 10 * p / (1.0 + (lk - 1) * p), dtype=torch.float64)
    want[77] /= p
    tolerance = (2 * half + rows / 2 * U + (d + 8) * U * (1.0 - 2.0 * score)) * 1.01 * want + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    if dtype == torch.float16:
        want[77] = math.inf                                                    # (2^25: more than the type holds)
    err = (dv[0, :, 0].double().cpu() - want).abs()
    err[77] = 0.0 if dtype == torch.float16 and bool(torch.isinf(dv[0, 77]).all()) else err[77]
    assert bool((err <= tolerance).all()), float((err / tolerance).max())
