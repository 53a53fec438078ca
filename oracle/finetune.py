"""Oracle of the fine-tuning operators, numpy in 64 bits, straight from the definitions in include/qrm.h: group norm with an
activation (Section 4.2's image decoder is made of such blocks) and its backward pass, one AdamW step with moments in 32 or 8 bits, the
message loss of Section 4.1 with its gradient."""
from __future__ import annotations

import numpy as np

BLOCK = 256


def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1.0 + e)


def _act(z, act):
    if act == "relu":
        return np.where(z < 0, 0.0, z)
    return z * _sigmoid(z) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return np.where(z <= 0, 0.0, 1.0)
    if act == "silu":
        s = _sigmoid(z)
        return s + z * s * (1.0 - s)
    return np.ones_like(z)


def group_norm(x, gamma, beta, groups, act, eps):
    """x [N,P,C] -> y [N,P,C], mean [N,groups], rstd [N,groups]."""
    x = np.asarray(x, dtype=np.float64)
    n, p, c = x.shape
    xg = x.reshape(n, p, groups, c // groups)
    mean = xg.mean(axis=(1, 3))
    rstd = 1.0 / np.sqrt(((xg - mean[:, None, :, None]) ** 2).mean(axis=(1, 3)) + eps)
    h = ((xg - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(n, p, c)
    z = h * (1.0 if gamma is None else np.asarray(gamma, dtype=np.float64)) + (0.0 if beta is None else np.asarray(beta, dtype=np.float64))
    return _act(z, act), mean, rstd


def group_norm_backward(x, dy, gamma, beta, mean, rstd, groups, act):
    """-> dx [N,P,C], dgamma [C], dbeta [C]; mean and rstd as the forward pass left them."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    n, p, c = x.shape
    gamma = np.ones(c) if gamma is None else np.asarray(gamma, dtype=np.float64)
    beta = np.zeros(c) if beta is None else np.asarray(beta, dtype=np.float64)
    spread = lambda v: np.repeat(np.asarray(v, dtype=np.float64), c // groups, axis=1)[:, None, :]
    h = (x - spread(mean)) * spread(rstd)
    dz = dy * _act_slope(gamma * h + beta, act)
    over = lambda v: spread(v.reshape(n, p, groups, -1).mean(axis=(1, 3)))
    dx = spread(rstd) * (gamma * dz - over(gamma * dz) - h * over(gamma * dz * h))
    return dx, (dz * h).sum(axis=(0, 1)), dz.sum(axis=(0, 1))


def _blocks(v):
    v = np.asarray(v, dtype=np.float64).reshape(-1)
    return np.concatenate([v, np.zeros(-v.size % BLOCK)]).reshape(-1, BLOCK)


def pack_moment(which, value):
    """Codes (int8 of m, uint8 of the root of v) and f32 scales of a moment [n]; 64-bit arithmetic, scales rounded to 32 bits."""
    rows = _blocks(value if which == 0 else np.sqrt(np.asarray(value, dtype=np.float64)))
    n = np.asarray(value).size
    scale = np.abs(rows).max(axis=1).astype(np.float32)
    s = scale.astype(np.float64)[:, None]
    part = np.divide(np.abs(rows), s, out=np.zeros_like(rows), where=s > 0)
    if which == 0:
        code = (np.sign(rows) * np.minimum(np.rint(127.0 * np.sqrt(part)), 127)).astype(np.int8)
    else:
        code = np.maximum(np.minimum(np.rint(255.0 * np.sqrt(part)), 255), rows > 0).astype(np.uint8)
    return code.reshape(-1)[:n], scale


def unpack_moment(which, code, scale):
    c = np.asarray(code).astype(np.float64)
    s = np.repeat(np.asarray(scale, dtype=np.float64), BLOCK)[:c.size]
    return s * c * np.abs(c) / 127.0 ** 2 if which == 0 else (s * c * c / 255.0 ** 2) ** 2


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay=0.0, lr_scale=1.0, grad_scale=1.0):
    """-> p, m, v behind the step, 64 bits."""
    p, g, m, v = (np.asarray(t, dtype=np.float64) for t in (p, g, m, v))
    g = g * grad_scale
    lr = lr * lr_scale
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    return p * (1.0 - lr * weight_decay) - lr / (1.0 - beta1 ** step) * m / (np.sqrt(v) / np.sqrt(1.0 - beta2 ** step) + eps), m, v


def message_loss(logits, target, m, t, weight):
    """logits [N,bits], target [N,bits] or [bits] of 0/1 -> loss, gradient [N,bits], wrong bits [N], wrong symbols [N]."""
    z = np.asarray(logits, dtype=np.float64)
    n, bits = z.shape
    one = np.broadcast_to(np.asarray(target) != 0, z.shape)
    x = np.where(one, z, -z)
    bce = np.maximum(-x, 0.0) + np.log1p(np.exp(-np.abs(x)))
    right = np.exp(-bce.reshape(n, bits // m, m).sum(axis=2))
    over = np.maximum((1.0 - right).sum(axis=1) - t, 0.0)
    loss = bce.sum() / (n * bits) + weight / n * (over ** 2).sum()
    pull = 1.0 / (n * bits) + 2.0 * weight / n * over[:, None] * right
    grad = np.where(one, -1.0, 1.0) * _sigmoid(-x) * np.repeat(pull, m, axis=1)
    wrong = (z > 0) != one
    return loss, grad, wrong.sum(axis=1), wrong.reshape(n, bits // m, m).any(axis=2).sum(axis=1)
