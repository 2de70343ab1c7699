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


# ---- log-probabilities of labels and the clipped policy loss -------------------------------------
def logp_rows(z, labels):
    """z [rows, K] in 64 bits, labels [rows]: dict of t, l, logp, entropy, p, y, live and has (a label) for every row; a row
    left out has 0 in logp and entropy."""
    z, labels = np.asarray(z, F64), np.asarray(labels)
    K = z.shape[1]
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        t = np.where(np.isnan(z), -np.inf, z).max(1)
        has = (labels >= 0) & (labels < K)
        none = (z == -np.inf).all(1)
        y = z - np.where(np.isfinite(t), t, np.where(t == np.inf, np.inf, 0.0))[:, None]
        e = np.exp(y)
        s = e.sum(1)
        l = np.log(s)
        p = e / s[:, None]
        py = np.where(y == -np.inf, 0.0, p * np.where(y == -np.inf, 0.0, y))
        ent = l - py.sum(1)
        za = np.take_along_axis(z, np.where(has, labels, 0)[:, None], 1)[:, 0]
        logp = za - t - l
    live = has & ~none
    return dict(t=t, l=l, p=p, y=y, has=has, live=live, none=none, logp=np.where(live, logp, 0.0), entropy=np.where(live, ent, 0.0), za=za,
                s1=np.abs(py).sum(1), s2=np.where(y == -np.inf, 0.0, p * np.where(y == -np.inf, 0.0, y) ** 2).sum(1))


def logp_gradient(r, labels, dlogp, dent):
    """dlogits of rows (r: logp_rows) for given gradients of log-probability and entropy."""
    dlogp, dent = np.asarray(dlogp, F64), np.asarray(dent, F64)
    with np.errstate(invalid="ignore"):
        logq = r["y"] - r["l"][:, None]
        bonus = np.where(r["y"] == -np.inf, 0.0, r["p"] * (np.where(r["y"] == -np.inf, 0.0, logq) + r["entropy"][:, None]))
        d = -dlogp[:, None] * r["p"] - dent[:, None] * bonus
        np.put_along_axis(d, np.where(r["has"], labels, 0)[:, None],
                          np.take_along_axis(d, np.where(r["has"], labels, 0)[:, None], 1) + dlogp[:, None], 1)
    return d


def policy(z, labels, advantage, old, ref, weight, low, high, kl, entropy):
    """(out [4], dlogits [rows, K], logp, live, G) of the clipped policy loss; old, ref may be None."""
    r = logp_rows(z, labels)
    A, w = np.asarray(advantage, F64), np.asarray(weight, F64)
    live = r["live"] & (w != 0)
    with np.errstate(invalid="ignore", over="ignore"):
        ratio = np.exp(r["logp"] - old) if old is not None else np.ones_like(A)
        cut = ((A > 0) & (ratio > high)) | ((A < 0) & (ratio < low))
        gain = np.where(A == 0, 0.0, np.where(cut, np.clip(ratio, low, high), ratio) * A)
        loss, G, d, H = -gain, np.where(cut | (A == 0), 0.0, -ratio * A), np.zeros_like(A), np.zeros_like(A)
        if kl and ref is not None:
            q = ref - r["logp"]
            d = np.expm1(q) - q
            loss, G = loss + kl * d, G - kl * np.expm1(q)
        if entropy:
            H = r["entropy"]
            loss = loss - entropy * H
        out = np.array([(w * x)[live].sum() for x in (loss, d, H, cut.astype(F64))])
        dz = np.where(live[:, None], logp_gradient(r, labels, w * G, np.where(live, -entropy * w, 0.0)), 0.0)
    return out, dz, np.where(live, r["logp"], 0.0), live, G, ratio, r


# ---- Muon -------------------------------------------------------------------------------------------
NS = (3.4445, -4.7750, 2.0315)


def newton_schulz(u, steps=5, eps=1e-12):
    """The orthogonalised u, in 64 bits."""
    x = np.asarray(u, F64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (np.sqrt((x ** 2).sum()) + eps)
    for _ in range(steps):
        a = x @ x.T
        x = NS[0] * x + (NS[1] * a + NS[2] * a @ a) @ x
    return x.T if tall else x


def newton_schulz_fp16(u, steps=5, eps=1e-12):
    """The same with the roundings that the operator's definition allows: products of fp16 values (X, A off its diagonal, B off
    its diagonal), everything else in 64 bits."""
    def h(t, s):
        return (t * s).astype(np.float16).astype(F64) / s

    x = np.asarray(u, F64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (np.sqrt((x ** 2).sum()) + eps)
    for _ in range(steps):
        up = h(x, 2.0 ** 15)
        a = up @ up.T
        d = a.diagonal().copy()
        o = h(a - np.diag(d), 2.0 ** 15)
        q = (d[:, None] + d[None, :]) * o + o @ o
        e = NS[1] * d + NS[2] * (d * d + q.diagonal())
        b = h(NS[1] * o + NS[2] * (q - np.diag(q.diagonal())), 2.0 ** 14)
        x = (NS[0] + e)[:, None] * x + b @ up
    return x.T if tall else x


def muon(p, g, m, lr, mu, nesterov, weight_decay, scale, coef=1.0, steps=5, eps=1e-12, update=newton_schulz):
    """(p, m) after a step, and the update's matrix"""
    p, g, m = (np.asarray(a, F64) for a in (p, g, m))
    g = g * coef
    m = mu * m + g
    o = update(g + mu * m if nesterov else m, steps, eps)
    return p - lr * weight_decay * p - lr * scale * o, m, o
