"""How near attention in 32 bits is to 64 bits, as a whole: tolerances that arithmetic of fewer bits does not pass, which is shown on the CPU.

Of a norm over many elements roundings are counted as independent ones: n of them one behind the other move a sum by sqrt(n) halves of a unit in its last place, u = 2^-24
of what it is made of.  A score of D products of the usual spread (its summands' magnitudes are twice to three times the score's spread, for keys have a part that all rows
share) is off by 2 sqrt(D) u; a sum over n rows by sqrt(n) u; the product with the scale, the exponential's argument and result, the division and the results' rounding, and
numbers of up to 8 in the exponent, by 16 u.  Gradients have two such products behind each other, and a difference of two sums that are twice what is left: four times that.
"""
import math

import numpy as np
import pytest
import torch

from oracle import attention as at

U = 2.0 ** -24
# (images, queries, keys, heads, key heads, elements, causal): every kernel width and both sides of its borders, few rows, rows that are split
SHAPES = [(1, 61, 100, 2, 1, 16, False), (2, 60, 90, 2, 2, 32, True), (1, 70, 100, 4, 2, 40, False), (1, 64, 130, 2, 1, 64, True), (1, 90, 80, 2, 1, 72, False),
          (1, 50, 120, 2, 2, 96, True), (1, 129, 127, 2, 1, 128, False), (1, 70, 65, 2, 1, 136, True), (1, 60, 100, 2, 1, 200, False), (1, 100, 100, 1, 1, 256, True),
          (1, 60, 90, 1, 1, 264, False), (1, 128, 96, 2, 1, 512, False), (1, 3, 1000, 4, 1, 64, False), (2, 1, 900, 8, 2, 128, False), (1, 4, 700, 2, 1, 512, False)]


def allowed(shape):
    """-> (of o, of lse, of the gradients)"""
    n, lq, lk, heads, kv, d, causal = shape
    forward = U * (2.0 * math.sqrt(d) + math.sqrt(lk) + 16.0)
    return forward, forward, 4.0 * U * (2.0 * math.sqrt(d) + math.sqrt(lk + lq * heads // kv) + 16.0)


def inputs(shape):
    n, lq, lk, heads, kv, d, causal = shape
    r = np.random.default_rng(sum(shape))
    normal = lambda *s: r.normal(size=s).astype(np.float32)
    return [normal(n, lq, heads, d) * np.float32(1.4), normal(n, lk, kv, d) + normal(1, 1, kv, d) * np.float32(0.4), normal(n, lk, kv, d) + normal(1, 1, kv, d) * np.float32(0.7),
            normal(n, lq, heads, d) * np.float32(0.05)]


def away(got, want):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


def rounded(x, dtype):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(dtype).float().numpy()


def by_hand(shape, data, keep=np.float32, p_to=None, ds_to=None):
    """o, lse, dq, dk, dv image by image and head by head in `keep`, probabilities or score gradients rounded to a type of 16 bits."""
    n, lq, lk, heads, kv, d, causal = shape
    q, k, v, do = (t.astype(keep) for t in data)
    scale = keep(np.float32(d ** -0.5))
    o, lse, dq, dk, dv = np.zeros_like(q), np.zeros((n, heads, lq), keep), np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    seen = np.tril(np.ones((lq, lk), bool), lk - lq) if causal else np.ones((lq, lk), bool)
    some = seen.any(axis=1)
    to = lambda x, t: x if t is None else rounded(x, t).astype(keep)
    for i in range(n):
        for h in range(heads):
            g = h // (heads // kv)
            s = np.where(seen, (q[i, :, h] @ k[i, :, g].T) * scale, keep(-np.inf))
            top = np.where(some, s.max(axis=1), keep(0))
            e = np.exp(s - top[:, None])
            total = np.where(some, e.sum(axis=1), keep(1))
            lse[i, h] = np.where(some, top + np.log(total), keep(-np.inf))
            o[i, :, h] = (to(e, p_to) @ v[i, :, g]) / total[:, None]
            p = np.where(seen, np.exp(s - np.where(some, lse[i, h], keep(0))[:, None]), keep(0))
            ds = p * (do[i, :, h] @ v[i, :, g].T - (do[i, :, h] * o[i, :, h]).sum(axis=1, keepdims=True))
            dq[i, :, h] = scale * (to(ds, ds_to) @ k[i, :, g])
            dk[i, :, g] += scale * (to(ds, ds_to).T @ q[i, :, h])
            dv[i, :, g] += to(p, p_to).T @ do[i, :, h]
    return o, lse, dq, dk, dv


def exact(shape, data, o=None, lse=None):
    n, lq, lk, heads, kv, d, causal = shape
    scale = float(np.float32(d ** -0.5))
    want_o, want_lse, _ = at.attention(*data[:3], scale, causal)
    grads, _ = at.attention_backward(*data[:3], want_o if o is None else o, data[3], want_lse if lse is None else lse, scale, causal)
    return want_o, want_lse, grads


def check(shape, data, got):
    o, lse, dq, dk, dv = got
    want_o, want_lse, grads = exact(shape, data, o, lse)
    far_o, far_lse, far_grads = allowed(shape)
    some = np.isfinite(want_lse)
    assert np.array_equal(some, np.isfinite(lse))
    found = dict(o=away(o, want_o) / far_o, lse=away(np.where(some, lse, 0.0), np.where(some, want_lse, 0.0)) / far_lse)
    found.update({name: away(a, b) / far_grads for name, a, b in zip(("dq", "dk", "dv"), (dq, dk, dv), grads)})
    return found


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_fewer_bits_do_not_pass(shape):
    """Planted in plain forms: 32 bits pass, P, dS or inputs of 16 bits are outside of what is allowed in each output that they reach."""
    data = inputs(shape)
    assert max(check(shape, data, by_hand(shape, data)).values()) <= 1.0
    for t in (torch.bfloat16, torch.float16):
        found = check(shape, data, by_hand(shape, data, np.float64, p_to=t))
        assert found["o"] > 1.0 and found["dv"] > 1.0, (t, found)
        found = check(shape, data, by_hand(shape, data, np.float64, ds_to=t))
        assert found["dq"] > 1.0 and found["dk"] > 1.0, (t, found)
        found = check(shape, data, by_hand(shape, [rounded(x, t) for x in data], np.float64))
        assert min(found.values()) > 1.0, (t, found)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_f32_has_32_bits(shape):
    import paper_2509_02447_amd as qrm
    n, lq, lk, heads, kv, d, causal = shape
    data = inputs(shape)
    q, k, v, do = (torch.from_numpy(x).cuda() for x in data)
    o, lse, dq, dk, dv = torch.empty_like(q), torch.empty((n, heads, lq), device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ctx = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
    desc = qrm.attention_desc(n, lq, lk, heads, kv, d, torch.float32, causal)
    ctx.qrm_attention(desc, q, k, v, o, lse)
    ctx.qrm_attention_backward(desc, q, k, v, o, do, lse, dq, dk, dv)
    torch.cuda.synchronize()
    found = check(shape, data, [t.cpu().numpy() for t in (o, lse, dq, dk, dv)])
    ctx.close()
    assert max(found.values()) <= 1.0, found


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_16_bits_row_by_row(shape, dtype):
    """Each row against its own sums: a score's D + 8 roundings of the sum of |q| |k| of the row, half a step for each weight and for the result, f16 weights under 2^-14 in
    steps of 2^-24 where the largest is 2^11 and more (2^-36 of a row at most, each)."""
    import paper_2509_02447_amd as qrm
    n, lq, lk, heads, kv, d, causal = shape
    data = [rounded(x, dtype) for x in inputs(shape)]
    q, k, v, _ = (torch.from_numpy(x).cuda().to(dtype) for x in data)
    o, lse = torch.empty_like(q), torch.empty((n, heads, lq), device="cuda")
    ctx = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
    ctx.qrm_attention(qrm.attention_desc(n, lq, lk, heads, kv, d, dtype, causal), q, k, v, o, lse)
    torch.cuda.synchronize()
    scale, half = float(np.float32(d ** -0.5)), {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    want, want_lse, weight = at.attention(*data[:3], scale, causal)
    a = [np.abs(x.astype(np.float64)) for x in data]
    size = np.stack([(scale * np.einsum("nid,njd->nij", a[0][:, :, h], a[1][:, :, h // (heads // kv)])).max(axis=2) for h in range(heads)], axis=2)[..., None]  # [n, lq, heads, 1]
    scores = (d + 8) * U * (1.0 + 2.0 * size)
    tol = (half + 2 * scores + (2 * lk + 32) * U) * weight * 1.01 + half * np.abs(want) + 2.0 ** -24
    if dtype == torch.float16:
        tol += lk * 2.0 ** -36 * a[2].max()
    assert (np.abs(o.double().cpu().numpy() - want) <= tol).all()
    got, some = lse.double().cpu().numpy(), np.isfinite(want_lse)
    assert np.array_equal(some, np.isfinite(got))
    far = np.moveaxis(scores[..., 0], 1, 2) + (lk + 16) * U + 4 * U * np.abs(want_lse)
    assert (np.abs(got - want_lse)[some] <= far[some]).all()
    ctx.close()
