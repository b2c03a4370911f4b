"""Plain numpy fp64 forms of attention over selected blocks of keys and of what feeds it (axis rotations, means over blocks, the
choice of blocks), written from their definitions. Test infrastructure only."""
import numpy as np

BQ, BK = 128, 64


def rope_axes(x, gain, norm, H, dh, pos, freq, axis, halves, out_scale=1.0):
    """x [L, H*dh] -> [H, L, dh]; norm "none", "width" or "head"; pair p turns by pos[:, axis[p]] * freq[p]."""
    x = np.asarray(x, np.float64)
    L = x.shape[0]
    if norm == "width":
        x = x / np.sqrt(np.mean(x * x, 1, keepdims=True) + 1e-6) * gain
    x = x.reshape(L, H, dh)
    if norm == "head":
        x = x / np.sqrt(np.mean(x * x, 2, keepdims=True) + 1e-6) * gain
    y = x.copy()
    n = len(freq)
    for p in range(n):
        if not 0 <= axis[p] < pos.shape[1]:
            continue
        a, b = (p, n + p) if halves else (2 * p, 2 * p + 1)
        t = pos[:, axis[p]].astype(np.float64) * freq[p]
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        y[:, :, b] = x[:, :, a] * s + x[:, :, b] * c
    return (y * out_scale).transpose(1, 0, 2)


def block_mean(X, L, block):
    """X [H, Lpad, dh] -> [H, ceil(L / block), dh]."""
    X = np.asarray(X, np.float64)
    return np.stack([X[:, a:min(a + block, L)].mean(1) for a in range(0, L, block)], 1)


def block_select(Qm, Km, keep, rule=None):
    """Qm [H, nq, dh], Km [Hk, nk, dh] -> int32 [H, nq, keep]: first by class, score, index; ascending, -1 behind."""
    Qm, Km = np.asarray(Qm, np.float64), np.asarray(Km, np.float64)
    H, nq, _ = Qm.shape
    Hk, nk, _ = Km.shape
    cls = np.zeros(nk, int) if rule is None else np.where(rule == 1, 0, np.where(rule == 2, 2, 1))
    out = np.full((H, nq, keep), -1, np.int32)
    for h in range(H):
        for a in range(nq):
            with np.errstate(invalid="ignore"):
                s = Km[h // (H // Hk)] @ Qm[h, a]
            order = sorted((b for b in range(nk) if cls[b] != 2),
                           key=lambda b: (cls[b], -s[b] if s[b] == s[b] else np.inf, s[b] != s[b], b))
            best = sorted(order[:keep])
            out[h, a, :len(best)] = best
    return out


def attention_blocks(Q, K, V, blocks, Lq, Lk, log2_queries=False):
    """Q [H, >= Lq, dh], K and V [Hk, >= Lk, dh], blocks [H, nq, keep] -> (O [Lq, H*dh], the same with |V| for V: how large the
    weighted values are, which is what roundings of the weights are relative to)."""
    H, _, dh = Q.shape
    Hk = K.shape[0]
    nk = -(-Lk // BK)
    O, A = np.zeros((Lq, H, dh)), np.zeros((Lq, H, dh))
    for h in range(H):
        k, v = K[h // (H // Hk)].astype(np.float64), V[h // (H // Hk)].astype(np.float64)
        for a in range(-(-Lq // BQ)):
            rows = slice(a * BQ, min((a + 1) * BQ, Lq))
            seen = [np.arange(b * BK, min((b + 1) * BK, Lk)) for b in blocks[h, a] if 0 <= b < nk]
            if not seen:
                continue
            seen = np.concatenate(seen)
            z = Q[h, rows].astype(np.float64) @ k[seen].T * (np.log(2.0) if log2_queries else 1 / np.sqrt(dh))
            top = z.max(1, keepdims=True)
            w = np.exp(z - np.where(np.isinf(top), 0.0, top))
            total = w.sum(1, keepdims=True)
            w = w / np.where(total > 0, total, 1.0)
            O[rows, h], A[rows, h] = w @ v[seen], w @ np.abs(v[seen])
    return O.reshape(Lq, H * dh), A.reshape(Lq, H * dh)
