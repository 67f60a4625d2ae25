"""Plain 64-bit definitions, on the CPU, of the operators that train on answers, drop elements and serve in four bits."""
import math

import numpy as np
import torch

INF = math.inf
FP32_MOST = 2.0 ** 128 - 2.0 ** 103       # from here on a number rounds to infinity in fp32


def log_softmax_row(z):
    """(log probabilities, probabilities) of one row in float64; a row of -inf: -inf and 0"""
    top = z.max()
    if bool(torch.isnan(z).any()) or top == INF:
        return torch.full_like(z, math.nan), torch.full_like(z, math.nan)
    if top == -INF:
        return torch.full_like(z, -INF), torch.zeros_like(z)
    l = (z - top) - torch.log(torch.exp(z - top).sum())       # (top + log would lose the log beside a top of 1e38)
    return l, torch.exp(l)


def policy_loss(z, drawn, old, ref, advantage, weights, low, high, kl, scale):
    """(loss, log_prob, grad, factor) in float64; old, ref: lists of floats or None.  factor: the row's d (scale loss) / d log_prob"""
    n, c = z.shape
    loss, logs, grad, factor = [0.0] * n, [0.0] * n, torch.zeros(n, c, dtype=torch.float64), [0.0] * n
    for i in range(n):
        a, r, A = int(drawn[i]), float(weights[i]), float(advantage[i])
        if a < 0 or r == 0:
            continue
        lp, p = log_softmax_row(z[i])
        l = float(lp[a]) if a < c else math.nan
        logs[i] = l
        if math.isnan(l):
            loss[i] = math.nan
            grad[i] = math.nan
            factor[i] = math.nan
            continue
        lost = l == -INF
        ratio = 0.0 if lost else 1.0 if old is None else math.exp(min(l - old[i], 709.0)) if l - old[i] < 709 else INF
        free = 0.0 if A == 0 else ratio * A
        held = min(max(ratio, 1 - low), 1 + high) * A if A != 0 else 0.0
        value, slope = (-held, 0.0) if free > held else (-free, -free)
        if kl:
            gap = 0.0 if lost and ref[i] == -INF else ref[i] - l
            e = math.expm1(gap) if gap < 709 else INF
            value += kl * (INF if gap == INF else e - gap)
            slope -= kl * e
        loss[i] = r * value
        if lost or abs(loss[i]) > FP32_MOST:
            continue
        f = scale * r * slope
        factor[i] = f
        grad[i] = -f * p
        grad[i, a] += f
    return torch.tensor(loss, dtype=torch.float64), torch.tensor(logs, dtype=torch.float64), grad, torch.tensor(factor, dtype=torch.float64)


def pair_loss(h, hinge):
    if math.isnan(h):
        return math.nan, math.nan
    if hinge:
        return max(0.0, 1 - h), -1.0 if h < 1 else 0.0
    e = math.exp(-abs(h))
    return max(-h, 0.0) + math.log1p(e), -(e if h >= 0 else 1.0) / (1 + e)


def preference_loss(z, labels, ends, ref, weights, pair_weights, hinge, beta, eps, scale):
    """(loss, margin, grad, per-pair slopes) in float64"""
    n, c = z.shape
    pairs = len(ends) // 2
    gain = [0.0] * n
    probs = [None] * n
    for i in range(n):
        a, r = int(labels[i]), float(weights[i])
        if a < 0 or r == 0 or not ends[0] <= i < ends[-1]:
            continue
        lp, probs[i] = log_softmax_row(z[i])
        l = float(lp[a]) if a < c else math.nan
        gain[i] = 0.0 if l == -INF and ref[i] == -INF else r * (l - ref[i])
    loss, margin, slopes, grad = [], [], [], torch.zeros(n, c, dtype=torch.float64)
    for p in range(pairs):
        a, b, e = ends[2 * p:2 * p + 3]
        h = beta * (sum(gain[a:b]) - sum(gain[b:e]))
        L, d = pair_loss(h, hinge)
        if eps:
            L2, d2 = pair_loss(-h, hinge)
            L, d = (1 - eps) * L + eps * L2, (1 - eps) * d - eps * d2
        w = float(pair_weights[p])
        loss.append(w * L if w else 0.0)
        margin.append(h)
        slopes.append(d)
        if w == 0:
            continue
        for i in range(a, e):
            if probs[i] is None:
                continue
            f = scale * beta * w * d * float(weights[i]) * (1 if i < b else -1)
            empty = bool((z[i] == -INF).all())
            if f != 0 and not empty:
                grad[i] = -f * probs[i]
                if int(labels[i]) < c:
                    grad[i, int(labels[i])] += f
    make = lambda v: torch.tensor(v, dtype=torch.float64)  # noqa: E731
    return make(loss), make(margin), grad, make(slopes)


def philox(counter, key):
    """Philox4x32-10 of one counter, in Python's whole numbers"""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def drop_bits(n, d, seed, chain, step):
    """the sixteen bits of every element, n x d"""
    blocks = -(-d // 8)
    u = np.uint64
    c = [np.tile(np.arange(blocks, dtype=u), n), np.repeat(np.arange(n, dtype=u), blocks), np.full(n * blocks, chain, dtype=u),
         np.full(n * blocks, (1 << 30) + step % (1 << 30), dtype=u)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & u(0xFFFFFFFF), (a >> u(32)) ^ c[3] ^ u(k[1]), a & u(0xFFFFFFFF)]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    halves = [(w >> u(s)) & u(0xFFFF) for w in c for s in (0, 16)]
    return np.stack(halves, 1).reshape(n, 8 * blocks)[:, :d].astype(np.int64)


FOUR = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def quantize4(x, group):
    """(codes n x whole blocks of 128 in the columns' order, scales n x groups in float64) of a float64 matrix that holds fp32 values"""
    n, d = x.shape
    blocks = -(-d // 128)
    y = np.zeros((n, blocks * 128))
    y[:, :d] = x
    y = y.reshape(n, -1, group)
    fine = np.isfinite(y).all(-1)
    top = np.where(fine, np.abs(np.where(np.isfinite(y), y, 0)).max(-1), 0.0)
    scales = np.ones_like(top)
    for i, j in zip(*np.nonzero(top)):
        # the least number of eight significant bits whose sixfold reaches the top
        _, e = math.frexp(top[i, j] / 6)
        unit = 2.0 ** (e - 8)
        m = math.ceil(top[i, j] / (6 * unit))
        while 6 * (m - 1) * unit >= top[i, j]:
            m -= 1
        while 6 * m * unit < top[i, j]:
            m += 1
        scales[i, j] = max(m * unit, 2.0 ** -126)
    v = np.where(np.isfinite(y), y, 0) / scales[..., None]
    size = np.abs(v)
    hi = np.searchsorted(FOUR[:8], size).clip(1, 7)
    up, down = FOUR[hi] - size, size - FOUR[hi - 1]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    code = np.where(size >= 6, 7, code) + np.where(np.signbit(v), 8, 0)
    code = np.where(fine[..., None], code, 0)
    scales = np.where(fine, scales, math.nan)
    scales[:, -(-d // group):] = 0
    return code.reshape(n, blocks * 128).astype(np.uint8), scales


def pack4(code):
    """codes in the columns' order, whole blocks, to bytes in the blocks' own"""
    n, w = code.shape
    out = np.zeros((n, w // 2), dtype=np.uint8)
    for c in range(w):
        b, c128 = c // 128, c % 128
        j, k, e = c128 // 32, c128 % 32 // 8, c128 % 8
        out[:, 64 * b + 16 * k + 4 * j + e // 2] |= code[:, c] << (4 * (e % 2))
    return out


def values4(code, scales, group, d):
    n = code.shape[0]
    return (FOUR[code].reshape(n, -1, group) * scales[:, :code.shape[1] // group, None]).reshape(n, -1)[:, :d]
