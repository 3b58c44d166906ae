"""The router (include/brgemm.h) in numpy and 64 bits, row by row from its definition."""
import numpy as np


def softmax(x):
    with np.errstate(invalid="ignore"):
        m = np.where(np.isnan(x), -np.inf, x).max()
        if m == -np.inf:
            return np.zeros_like(x)
        p = np.exp(x - m)
        return p / p.sum()


def route(x, topk, valid=None, level=False):
    M, E = x.shape
    ids, gates = np.full((M, topk), -1, np.int64), np.zeros((M, topk))
    p = np.zeros((M, E))
    for t in range(M):
        if valid is not None and not valid[t]:
            continue
        p[t] = softmax(x[t])
        able = [e for e in range(E) if not np.isnan(x[t, e]) and x[t, e] > -np.inf]
        best = sorted(able, key=lambda e: (-x[t, e], e))[:topk]
        ids[t, :len(best)] = best
        g = p[t, best]
        gates[t, :len(best)] = g / g.sum() if level and len(best) else g
    counted = ids[:, 0] >= 0
    counts = np.array([(ids == e).sum() for e in range(E)])
    offsets = np.concatenate([[0], counts.cumsum()])
    rows, place = np.full(M * topk, -1, np.int64), np.full((M, topk), -1, np.int64)
    at = offsets[:-1].copy()
    for t in range(M):
        for j in range(topk):
            if ids[t, j] >= 0:
                place[t, j] = at[ids[t, j]]
                rows[at[ids[t, j]]] = t
                at[ids[t, j]] += 1
    n = counted.sum()
    mean = p[counted].sum(0) / n if n else np.zeros(E)
    share = counts / max(1, counts.sum())
    return dict(ids=ids, gates=gates, offsets=offsets, rows=rows, place=place, p=p,
                balance=np.concatenate([[E * (share * mean).sum(), n], mean]))


def value(x, ids, share, dgates, dloss, level):
    """What gemm_route_grad is the gradient of, with the choice and the shares held."""
    M, E = x.shape
    total, means, n = 0.0, np.zeros(E), 0
    for t in range(M):
        at = [e for e in ids[t] if e >= 0]
        if not at:
            continue
        p = softmax(x[t])
        n += 1
        means += p
        g = p[at] / (p[at].sum() if level else 1.0)
        total += (g * dgates[t, :len(at)]).sum()
    return total + (dloss * E * (share * means).sum() / n if n else 0.0)


def gradient(x, ids, share, dgates, dloss, level):
    M, E = x.shape
    out = np.zeros((M, E))
    n = (ids >= 0).any(1).sum()
    for t in range(M):
        chosen = ids[t] >= 0
        at = ids[t][chosen]
        if not len(at):
            continue
        p = softmax(x[t])
        d = np.zeros(E)
        d[at] = dgates[t][chosen]
        v = p
        if level:
            v = np.zeros(E)
            v[at] = p[at] / p[at].sum()
        out[t] = v * (d - (v * d).sum()) + dloss * E / n * p * (share - (p * share).sum())
    return out
