"""Plain 64-bit implementations of the training operators (include/unettrain.h): the reference of their tests.

Maps are [N, C, P] whatever their order in memory.  Two decisions are taken in fp32, as the operators' definition says:
on which side of a ReLU's kink an element lies (z formed with every operation rounded by itself), and the hash behind the
stochastic rounding.
"""
from __future__ import annotations

import numpy as np

F32, F64 = np.float32, np.float64


def _grouped(x, groups):
    return np.asarray(x, dtype=F64).reshape(x.shape[0], groups, -1)


def groupnorm_stats(x, groups, eps):
    g = _grouped(x, groups)
    mean = g.mean(2)
    return mean, 1 / np.sqrt(((g - mean[..., None]) ** 2).mean(2) + eps)


def _sigmoid(z):
    return 0.5 * (1 + np.tanh(0.5 * z))


def groupnorm_fwd(x, gamma, beta, groups, eps, act):
    """(y, mean, rstd)"""
    N, C, P = x.shape
    mean, rstd = groupnorm_stats(x, groups, eps)
    xh = ((_grouped(x, groups) - mean[..., None]) * rstd[..., None]).reshape(N, C, P)
    z = xh * np.asarray(gamma, F64)[None, :, None] + np.asarray(beta, F64)[None, :, None]
    y = {"none": lambda: z, "relu": lambda: np.where(z <= 0, 0.0, z), "silu": lambda: z * _sigmoid(z)}[act]()
    return y, mean, rstd


def groupnorm_bwd(x, dy, gamma, beta, mean, rstd, groups, act):
    """(dx, dgamma, dbeta) for given statistics; x fp32 or bf16 values as fp32."""
    N, C, P = x.shape
    per = C // groups
    ga, be = np.asarray(gamma, F64)[None, :, None], np.asarray(beta, F64)[None, :, None]
    mu, r = (np.repeat(np.asarray(t, F64), per, axis=1)[..., None] for t in (mean, rstd))
    xh = (np.asarray(x, F64) - mu) * r
    z = xh * ga + be
    dz = np.asarray(dy, F64)
    if act == "relu":
        z32 = (x.astype(F32) - mu.astype(F32)) * r.astype(F32) * ga.astype(F32) + be.astype(F32)
        assert z32.dtype == F32
        dz = np.where(z32 > 0, dz, np.where(z32 <= 0, 0.0, np.nan))
    elif act == "silu":
        s = _sigmoid(z)
        dz = dz * s * (1 + z * (1 - s))
    t = dz * ga
    tg, xg = _grouped(t, groups), _grouped(xh, groups)
    dx = (tg - tg.mean(2, keepdims=True) - xg * (tg * xg).mean(2, keepdims=True)).reshape(N, C, P) * r
    return dx, (dz * xh).sum((0, 2)), dz.sum((0, 2))


def grad_norm(grads, max_norm):
    """(norms, norm, coef)"""
    norms = np.array([np.sqrt((np.asarray(g, F64) ** 2).sum()) for g in grads])
    norm = np.sqrt((norms ** 2).sum())
    return norms, norm, 1.0 if norm == 0 else min(1.0, max_norm / norm)


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay, coef=1.0):
    """(p, m, v) after step number t"""
    p, g, m, v = (np.asarray(a, F64) for a in (p, g, m, v))
    g = g * coef
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    step = lr / (1 - beta1 ** t) * m / (np.sqrt(v) / np.sqrt(1 - beta2 ** t) + eps)
    return p - lr * weight_decay * p - step, m, v


def e4m3(codes):
    """Values of OCP e4m3 bytes."""
    c = np.asarray(codes, np.int64)
    e, f = (c >> 3) & 15, c & 7
    val = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where((c & 127) == 127, np.nan, np.where(c & 128, -val, val))


def block_exponents(x):
    """e of every block of 32: the smallest (from -127 on) with |x| <= 448 * 2^e."""
    top = np.abs(np.asarray(x, F64)).reshape(-1, 32).max(1)
    e = np.full(top.shape, -127)
    pos = top > 0
    e[pos] = np.maximum(-127, np.ceil(np.log2(top[pos] / 448)))
    # log2 may land on the wrong side of a power of two
    e = np.where(top > 448 * 2.0 ** e, e + 1, e)
    return np.where((e > -127) & (top <= 448 * 2.0 ** (e - 1)), e - 1, e)


def grid_step(q):
    """Distance of the e4m3 values around |q|."""
    return 2.0 ** (np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -6))) - 3)


def random16(position, t, seed):
    """The sixteen bits (as a fraction of one) that round the state at each position in step t."""
    with np.errstate(over="ignore"):
        x = (np.asarray(position, np.uint64) >> np.uint64(1)).astype(np.uint32) + np.uint32((seed + t * 0x9E3779B9) & 0xFFFFFFFF)
        x = (x ^ (x >> np.uint32(16))) * np.uint32(0x9E3779B9)
        x = (x ^ (x >> np.uint32(15))) * np.uint32(0x6A09E667)
        x = x ^ (x >> np.uint32(16))
    return np.where(np.asarray(position) % 2 == 0, x & np.uint32(0xFFFF), x >> np.uint32(16)) / 65536.0
