"""Pins of the fine-tuning oracle: worked values, invariants, and every gradient against differences of the forward definition."""
import numpy as np
import pytest

from oracle import finetune as ft


def _norm_inputs(seed, n=2, p=5, c=12):
    g = np.random.default_rng(seed)
    return g.normal(1.0, 2.0, (n, p, c)), g.normal(1.0, 0.3, c), g.normal(0.0, 0.3, c), g.normal(0.0, 1.0, (n, p, c))


def test_group_norm_worked_values():
    x = np.array([[[1.0, 3.0], [5.0, 7.0]]])                 # one group: mean 4, variance 5
    y, mean, rstd = ft.group_norm(x, None, None, 1, "none", 4.0)
    assert mean[0, 0] == 4.0 and rstd[0, 0] == pytest.approx(1 / 3)
    assert np.allclose(y, [[[-1.0, -1 / 3], [1 / 3, 1.0]]])
    assert np.array_equal(ft.group_norm(x, None, None, 1, "relu", 4.0)[0] == 0, y < 0)
    z = y[0, 1, 1]
    assert ft.group_norm(x, None, None, 1, "silu", 4.0)[0][0, 1, 1] == pytest.approx(z / (1 + np.exp(-z)))


@pytest.mark.parametrize("groups", [1, 3, 12])
def test_group_norm_leaves_every_group_with_mean_zero_and_variance_one(groups):
    x, *_ = _norm_inputs(1)
    y = ft.group_norm(x, None, None, groups, "none", 1e-12)[0].reshape(2, 5, groups, -1)
    assert np.allclose(y.mean(axis=(1, 3)), 0) and np.allclose((y ** 2).mean(axis=(1, 3)), 1)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("groups", [1, 4])
def test_group_norm_gradients_against_differences(act, groups):
    x, gamma, beta, dy = _norm_inputs(2)
    f = lambda x, gamma, beta: float((ft.group_norm(x, gamma, beta, groups, act, 1e-3)[0] * dy).sum())
    _, mean, rstd = ft.group_norm(x, gamma, beta, groups, act, 1e-3)
    got = ft.group_norm_backward(x, dy, gamma, beta, mean, rstd, groups, act)
    for which, (value, grad) in enumerate(zip((x, gamma, beta), got)):
        for i in np.random.default_rng(3).choice(value.size, min(20, value.size), replace=False):
            args = [[x, gamma, beta], [x, gamma, beta]]
            for a, sign in zip(args, (1, -1)):
                a[which] = value.copy()
                a[which].reshape(-1)[i] += sign * 1e-6
            assert grad.reshape(-1)[i] == pytest.approx((f(*args[0]) - f(*args[1])) / 2e-6, rel=1e-5, abs=1e-6)


def test_adamw_first_step_moves_by_the_rate_against_the_sign():
    g = np.array([3.0, -0.2, 1e-3])
    p, m, v = ft.adamw(np.zeros(3), g, np.zeros(3), np.zeros(3), 1, 0.01, 0.9, 0.999, 0.0)
    assert np.allclose(p, -0.01 * np.sign(g)) and np.allclose(m, 0.1 * g) and np.allclose(v, 0.001 * g * g)
    p, _, _ = ft.adamw(np.full(3, 2.0), 0 * g, np.zeros(3), np.zeros(3), 1, 0.01, 0.9, 0.999, 1e-8, weight_decay=0.5)
    assert np.allclose(p, 2.0 * (1 - 0.005))
    a = ft.adamw(np.ones(3), g, g, g * g, 7, 0.01, 0.9, 0.99, 1e-8, lr_scale=0.5, grad_scale=0.25)
    b = ft.adamw(np.ones(3), 0.25 * g, g, g * g, 7, 0.005, 0.9, 0.99, 1e-8)
    assert all(np.array_equal(s, t) for s, t in zip(a, b))


@pytest.mark.parametrize("n", [1, 255, 256, 257, 1000])
def test_moments_in_8_bits(n):
    g = np.random.default_rng(n)
    m, v = g.normal(0, 1e-3, n), g.random(n) ** 4 * 1e-6
    for which, value, top in ((0, m, 127), (1, v, 255)):
        code, scale = ft.pack_moment(which, value)
        back = ft.unpack_moment(which, code, scale)
        root, kept = (np.abs(value), np.abs(back)) if which == 0 else (np.sqrt(value), np.sqrt(back))
        s = np.repeat(scale.astype(np.float64), ft.BLOCK)[:n]
        # nearest of codes whose roots are one apart: |sqrt(a) - sqrt(b)| <= half a step (a whole one where a root is kept above zero)
        assert (np.abs(np.sqrt(root / s) - np.sqrt(kept / s)) <= (0.5 + 0.5 * (np.abs(code.astype(int)) == 1) * which) / top + 1e-6).all()
        assert code.size == n and scale.size == -(-n // ft.BLOCK) and np.abs(code.astype(int)).max() == top
        if which == 1:
            assert ((value > 0) <= (code > 0)).all()
        assert np.array_equal(np.sign(back), np.sign(value) * (code != 0))


def test_moments_of_zero():
    for which in (0, 1):
        code, scale = ft.pack_moment(which, np.zeros(300))
        assert not code.any() and not scale.any() and not ft.unpack_moment(which, code, scale).any()


def test_message_loss_worked_values():
    # logits of zero: every bit log 2, a symbol of two bits is right with chance 1/4; three symbols, none corrected
    loss, grad, bits, symbols = ft.message_loss(np.zeros((1, 6)), np.array([1, 0, 1, 1, 0, 0]), 2, 0, 1.0)
    assert loss == pytest.approx(np.log(2) + 2.25 ** 2)
    assert np.allclose(np.abs(grad), 0.5 * (1 / 6 + 2 * 2.25 * 0.25)) and np.array_equal(grad[0] < 0, [1, 0, 1, 1, 0, 0])
    assert bits[0] == 3 and symbols[0] == 2                  # a logit of zero reads as 0
    assert ft.message_loss(np.zeros((1, 6)), np.ones(6), 2, 3, 1.0)[0] == pytest.approx(np.log(2))   # all three corrected


@pytest.mark.parametrize("m,t,weight", [(1, 0, 0.0), (4, 1, 1.0), (3, 0, 0.3), (2, 2, 5.0)])
def test_message_loss_gradient_against_differences(m, t, weight):
    g = np.random.default_rng(5)
    z, target = g.normal(0, 1.5, (3, 12)), g.integers(0, 2, (3, 12))
    grad = ft.message_loss(z, target, m, t, weight)[1]
    for i in range(z.size):
        up, down = z.copy(), z.copy()
        up.reshape(-1)[i] += 1e-6
        down.reshape(-1)[i] -= 1e-6
        d = (ft.message_loss(up, target, m, t, weight)[0] - ft.message_loss(down, target, m, t, weight)[0]) / 2e-6
        assert grad.reshape(-1)[i] == pytest.approx(d, rel=1e-5, abs=1e-9)


def test_message_loss_far_logits():
    z = np.array([[800.0, -800.0], [-800.0, 800.0]])
    loss, grad, bits, symbols = ft.message_loss(z, np.array([1, 0]), 2, 0, 1.0)
    assert loss == pytest.approx(1600 / 4 + 0.5) and np.array_equal(bits, [0, 2]) and np.array_equal(symbols, [0, 1])
    assert np.array_equal(grad[0], [0, 0]) and np.allclose(grad[1], [-0.25, 0.25])
