"""The oracle of attention against forms written another way: a softmax row by row, gradients by differences, the norm of known vectors."""
import numpy as np
import pytest

from oracle import attention as at


def inputs(seed, n=2, lq=5, lk=7, heads=4, kv=2, d=6):
    r = np.random.default_rng(seed)
    return r.normal(size=(n, lq, heads, d)), r.normal(size=(n, lk, kv, d)), r.normal(size=(n, lk, kv, d))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens", [(None, None), ([5, 3], [7, 2]), ([0, 9], [4, -1])])
def test_forward_row_by_row(causal, lens):
    q, k, v = inputs(1)
    o, lse, weight = at.attention(q, k, v, 0.3, causal, *lens)
    for n in range(2):
        a, b = (min(max(l[n], 0), m) if l else m for l, m in zip(lens, (5, 7)))
        for h in range(4):
            for i in range(5):
                keys = [j for j in range(b) if i < a and (not causal or j <= i + b - a)]
                if not keys:
                    assert np.isneginf(lse[n, h, i]) and not o[n, i, h].any()
                    continue
                e = [np.exp(0.3 * float(np.dot(q[n, i, h], k[n, j, h // 2]))) for j in keys]
                want = sum(x * v[n, j, h // 2] for x, j in zip(e, keys)) / sum(e)
                assert np.allclose(o[n, i, h], want) and np.isclose(lse[n, h, i], np.log(sum(e)))
                assert (weight[n, i, h] >= np.abs(o[n, i, h]) - 1e-12).all()


@pytest.mark.parametrize("causal", [False, True])
def test_backward_against_differences(causal):
    args = inputs(2)
    lens = ([5, 4], [7, 3])
    w = np.random.default_rng(3).normal(size=args[0].shape)
    o, lse, _ = at.attention(*args, 0.4, causal, *lens)
    grads, _ = at.attention_backward(*args, o, w, lse, 0.4, causal, *lens)
    r = np.random.default_rng(4)
    for index, g in enumerate(grads):
        for _ in range(20):
            where = tuple(r.integers(0, s) for s in g.shape)
            values = []
            for step in (1e-6, -1e-6):
                moved = [t.copy() for t in args]
                moved[index][where] += step
                values.append((at.attention(*moved, 0.4, causal, *lens)[0] * w).sum())
            assert np.isclose((values[0] - values[1]) / 2e-6, g[where], atol=1e-7)


def test_grad_norm():
    assert at.grad_norm([np.array([3.0]), None, np.array([[4.0]])], 10.0) == (5.0, 1.0)
    norm, scale = at.grad_norm([np.full(100, 2.0)], 5.0, 0.5)
    assert norm == 10.0 and scale == 0.25
