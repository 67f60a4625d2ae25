"""Plain 64-bit definitions of the many-class linear model's operators, on the CPU."""
import math

import numpy as np
import torch

INF = math.inf


def e4m3_values():
    """value of every code, from the format's definition: 4 exponent bits (bias 7), 3 mantissa bits, no infinity, 0x7f and 0xff NaN"""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        v[c] = math.nan if (c & 127) == 127 else -x if c >> 7 else x
    return v


E4M3 = e4m3_values()
_POSITIVE = E4M3[:127]


def nearest_code(v):
    """codes of the nearest e4m3 values, half to the even code; |v| <= 448"""
    s = np.abs(v)
    hi = np.searchsorted(_POSITIVE, s).clip(1, 126)
    lo = hi - 1
    up, down = _POSITIVE[hi] - s, s - _POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code + np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def quantize(x):
    """(codes, exps) of a float64 matrix, codes in whole blocks"""
    r, c = x.shape
    b = -(-c // 128)
    y = np.zeros((r, b * 128))
    y[:, :c] = x
    y = y.reshape(r, b, 128)
    s = np.where(np.isfinite(y), np.abs(y), 0).max(-1) if b else np.zeros((r, 0))
    e = np.zeros(s.shape, dtype=np.int64)
    for i, j in zip(*np.nonzero(s)):
        e[i, j] = math.frexp(s[i, j])[1] - 10
        while s[i, j] > 448 * 2.0 ** int(e[i, j]):
            e[i, j] += 1
    e = np.maximum(e, -126)
    with np.errstate(invalid="ignore"):
        v = y * 2.0 ** -e[..., None].astype(np.float64)
    codes = np.where(np.isfinite(y), nearest_code(np.where(np.isfinite(y), v, 0)), 127).astype(np.uint8)
    return codes.reshape(r, b * 128), (e + 127).astype(np.uint8)


def values(codes, exps):
    r, n = codes.shape
    return (E4M3[codes].reshape(r, n // 128, 128) * 2.0 ** (exps[:, :n // 128, None].astype(np.float64) - 127)).reshape(r, n)


def codes_of(q):
    """codes and exponents of a BlockMatrix as arrays"""
    return q.codes.view(torch.uint8).cpu().numpy(), q.exps.cpu().numpy()[:, :-(-q.cols // 128)]


def softmax_loss(z, labels, scale, weights):
    """(loss, grad) in float64"""
    n, c = z.shape
    loss, grad = torch.zeros(n, dtype=torch.float64), torch.zeros(n, c, dtype=torch.float64)
    for i in range(n):
        t, r = int(labels[i]), float(weights[i])
        if t < 0 or r == 0:
            continue
        if t >= c:
            loss[i] = math.nan
            grad[i] = math.nan
        elif bool((z[i] == -INF).all()):
            loss[i] = INF
        else:
            m = z[i].max()
            e = torch.exp(z[i] - m)
            loss[i] = r * (m + torch.log(e.sum()) - z[i, t])
            p = e / e.sum()
            p[t] -= 1
            grad[i] = scale * r * p
    return loss, grad


def draw(x, u, slope, top_k, top_p, min_p):
    """(class, q, Q) of one row by the definition, for scores whose weights 2^((x - max) slope) are exact in float64"""
    x = [-INF if v != v else float(v) for v in x]
    top = max(x)
    if top == -INF:
        return -1, 0, 1
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))
    e = [0.0 if v == -INF else 1.0 if v == top or slope is None else 2.0 ** ((v - top) * slope) for v in x]
    if slope is None:
        order = order[:1]
    elif top_k > 0:
        order = order[:top_k]
    q = [math.floor(v * 2 ** 31 + 0.5) for v in e]
    order = [i for i in order if e[i] >= min_p and x[i] != -INF]
    total = sum(q[i] for i in order)
    if top_p < 1:
        need, run, kept = min(max(math.ceil(float(top_p) * total), 1), total), 0, []
        for i in order:
            if run >= need:
                break
            kept.append(i)
            run += q[i]
        order = kept
        total = run
    target = min(int(float(u) * float(total)), total - 1)
    run = 0
    for i in sorted(order):
        run += q[i]
        if run > target:
            return i, q[i], total
    raise AssertionError
