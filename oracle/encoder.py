"""Plain numpy fp64 forms of a text encoder's operators (attention with a bias by distance, the gated feed-forward block, both with
their gradients) and of products of 8-bit integers, written from their definitions. Test infrastructure only."""
import math
from fractions import Fraction

import numpy as np


def quant_rows_i8(x):
    """Codes to the nearest of 127 x / max|x|, halves to even, and the scales max|x| / 127; rows that are not finite: codes 0, scale NaN."""
    x = np.asarray(x, np.float64)
    most = np.abs(x).max(1, keepdims=True)
    ok = np.isfinite(most) & (most > 0)
    with np.errstate(invalid="ignore", over="ignore"):
        codes = np.where(ok, np.rint(127.0 * x / np.where(ok, most, 1.0)), 0.0)
    return codes.astype(np.int8), np.where(np.isfinite(most), most / 127.0, np.nan)[:, 0]


def gelu(x):
    return 0.5 * x * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))


def gelu_slope(x):
    c = math.sqrt(2.0 / math.pi)
    t = np.tanh(c * (x + 0.044715 * x ** 3))
    return 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * x * x)


def silu(x):
    return x / (1.0 + np.exp(-x))


def silu_slope(x):
    s = 1.0 / (1.0 + np.exp(-x))
    return s * (1.0 + x * (1.0 - s))


ACT = {"gelu": (gelu, gelu_slope), "silu": (silu, silu_slope)}


def gated(x, w, act):
    """(h, both projections)."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    pre = x @ w.T
    F = w.shape[0] // 2
    return ACT[act][0](pre[:, :F]) * pre[:, F:], pre


def gated_backward(x, w, pre, dh, act):
    """(dx, dw, gradient of the projections)."""
    x, w, pre, dh = (np.asarray(t, np.float64) for t in (x, w, pre, dh))
    F = w.shape[0] // 2
    a, slope = ACT[act]
    d = np.concatenate((dh * pre[:, F:] * slope(pre[:, :F]), dh * a(pre[:, :F])), 1)
    return d @ w, d.T @ x, d


def bias_buckets(n_buckets, far, both_sides):
    """Bucket of each distance key - query from -far to far, in exact arithmetic: one each for the nearest, then logarithmic steps."""
    side = n_buckets // 2 if both_sides else n_buckets
    near = side // 2

    def of(n):
        if n < near:
            return n
        k = 0
        while k + 1 < side - near and Fraction(n, near) ** (side - near) >= Fraction(far, near) ** (k + 1):
            k += 1
        return near + k

    if both_sides:
        return np.array([of(abs(d)) + (side if d > 0 else 0) for d in range(-far, far + 1)], np.int32)
    return np.array([of(max(0, -d)) for d in range(-far, far + 1)], np.int32)


def attention_bias(q, k, v, table, bucket, lens, first, causal, scale):
    """q [B, Lq, H, dh], k and v [B, Lk, Hk, dh] -> (o [B, Lq, H, dh], lse [B, H, Lq], probabilities [B, H, Lq, Lk])."""
    q, k, v, table = (np.asarray(t, np.float64) for t in (q, k, v, table))
    B, Lq, H, dh = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    R = (len(bucket) - 1) // 2
    o, lse, P = np.zeros(q.shape), np.full((B, H, Lq), -np.inf), np.zeros((B, H, Lq, Lk))
    for b in range(B):
        at = np.arange(Lk)[None] - np.arange(Lq)[:, None] - int(first[b])
        see = np.broadcast_to(np.arange(Lk)[None] < lens[b], at.shape)
        if causal:
            see = see & (at <= 0)
        of = np.asarray(bucket)[np.clip(at, -R, R) + R]
        for h in range(H):
            s = np.where(see, (q[b, :, h] @ k[b, :, h // (H // Hk)].T) * scale + table[of, h], -np.inf)
            m = s.max(1, initial=-np.inf)
            p = np.exp(s - np.where(np.isfinite(m), m, 0.0)[:, None])
            total = p.sum(1)
            some = total > 0
            P[b, h] = p / np.where(some, total, 1.0)[:, None]
            lse[b, h] = np.where(some, m + np.log(np.where(some, total, 1.0)), -np.inf)
            o[b, :, h] = P[b, h] @ np.where((np.arange(Lk) < lens[b])[:, None], v[b, :, h // (H // Hk)], 0.0)
    return o, lse, P


def attention_bias_backward(q, k, v, table, bucket, lens, first, causal, scale, do):
    """dq, dk, dv, dtable of sum(o * do), and the sums of magnitudes that their errors are measured by."""
    o, _, P = attention_bias(q, k, v, table, bucket, lens, first, causal, scale)
    q, k, v, do = (np.asarray(t, np.float64) for t in (q, k, v, do))
    B, Lq, H, dh = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    R = (len(bucket) - 1) // 2
    dq, dk, dv, dtable = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(np.shape(table))
    mq, mk, mv, mt = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(np.shape(table))
    for b in range(B):
        of = np.asarray(bucket)[np.clip(np.arange(Lk)[None] - np.arange(Lq)[:, None] - int(first[b]), -R, R) + R]
        for h in range(H):
            g = h // (H // Hk)
            p, d = P[b, h], do[b, :, h]
            dp = d @ v[b, :, g].T
            delta = (p * dp).sum(1, keepdims=True)
            ds = p * (dp - delta)
            # what the products and the subtraction are made of
            size = p * (np.abs(d) @ np.abs(v[b, :, g]).T + np.abs(d * o[b, :, h]).sum(1, keepdims=True))
            dq[b, :, h] = ds @ k[b, :, g] * scale
            dk[b, :, g] += ds.T @ q[b, :, h] * scale
            dv[b, :, g] += p.T @ d
            np.add.at(dtable[:, h], of.ravel(), ds.ravel())
            a = np.abs(ds) + 2.0 ** -6 * size
            # in the products for dq delta has the roundings of o's weights in it, to 8 bits
            row = (np.abs(d) * (p @ np.abs(v[b, :, g]))).sum(1, keepdims=True)
            mq[b, :, h] = (a + p * row) @ np.abs(k[b, :, g]) * scale
            mk[b, :, g] += a.T @ np.abs(q[b, :, h]) * scale
            mv[b, :, g] += p.T @ np.abs(d)
            np.add.at(mt[:, h], of.ravel(), size.ravel())
    return (dq, dk, dv, dtable), (mq, mk, mv, mt)
