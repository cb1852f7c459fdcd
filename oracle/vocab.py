"""64-bit implementations of the vocabulary operators, row by row in numpy, from their definitions: the top logits of
a row, distillation from a teacher's top logits, and the drawing of a token.

All take float64 arrays that hold the exact bf16 or fp32 values.
"""
import numpy as np


def _selectable(z):
    return ~np.isnan(z) & (z > -np.inf)


def descending(z):
    """Indices of a row's selectable logits: descending values, ties by the lower index."""
    at = np.flatnonzero(_selectable(z))
    return at[np.argsort(-z[at], kind="stable")]


def top_logits(z, K):
    """(values [T][K], idx [T][K]); -inf and -1 where a row has fewer selectable logits."""
    T = z.shape[0]
    values, idx = np.full((T, K), -np.inf), np.full((T, K), -1, np.int64)
    for r in range(T):
        o = descending(z[r])[:K]
        values[r, :o.size], idx[r, :o.size] = z[r, o], o
    return values, idx


def _lse(x):
    with np.errstate(all="ignore"):
        m = np.max(x)
        return m + np.log(np.sum(np.exp(x - m))) if np.isfinite(m) else (np.nan if np.isnan(x).any() or m > 0 else m)


def teacher_shares(V, idx, val, tau):
    """(indices, shares) of a row's present entries; empty if none has a weight."""
    ok = (idx >= 0) & (idx < V) & (val > -np.inf)
    i, t = idx[ok], val[ok] / tau
    if i.size == 0:
        return i, t
    q = np.exp(t - t.max())
    return i, q / q.sum()


def distill(z, idx, val, labels, tau, alpha, g=None):
    """(loss [T], lse [T][2], dlogits [T][V]); a label outside [0, V) makes its row an ignored one."""
    T, V = z.shape
    loss, lse, d = np.zeros(T), np.zeros((T, 2)), np.zeros((T, V))
    for r in range(T):
        y = None if labels is None else int(labels[r])
        if y is not None and not 0 <= y < V:
            continue
        lse[r] = _lse(z[r] / tau), _lse(z[r])
        i, q = (np.zeros(0, np.int64), np.zeros(0)) if idx is None else teacher_shares(V, idx[r], val[r], tau)
        with np.errstate(invalid="ignore"):
            if alpha > 0 and i.size:
                live = q > 0
                logp = z[r, i[live]] / tau - lse[r, 0]
                loss[r] += alpha * tau ** 2 * np.sum(q[live] * (np.log(q[live]) - logp))
                d[r] += alpha * tau * np.exp(z[r] / tau - lse[r, 0])
                np.subtract.at(d[r], i, alpha * tau * q)
            if alpha < 1 and y is not None:
                loss[r] += (1 - alpha) * (lse[r, 1] - z[r, y])
                d[r] += (1 - alpha) * np.exp(z[r] - lse[r, 1])
                d[r, y] -= 1 - alpha
        if g is not None:
            d[r] *= g[r]
    return loss, lse, d


def sample(z, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """(ids, logprob, n_kept, margin) per row.  margin: how far, relative to the mass it is measured by, the nearest
    decision (the nucleus, the drawn token) is from going the other way; infinite where all weights are 0 or 1, whose
    sums and products with a 24-bit number are exact on both sides."""
    B, V = z.shape
    ids, logprob, n_kept, margin = np.full(B, -1), np.full(B, -np.inf), np.zeros(B, np.int64), np.full(B, np.inf)
    for r in range(B):
        T = 1.0 if temperature is None else float(temperature[r])
        k = 0 if top_k is None else int(top_k[r])
        p = 1.0 if top_p is None else float(top_p[r])
        mp = 0.0 if min_p is None else float(min_p[r])
        if not 0 <= T < np.inf or np.isnan(p) or not mp <= 1 or not 0 <= u[r] < 1:
            logprob[r] = np.nan
            continue
        o = descending(z[r])
        if o.size == 0:
            continue
        if T == 0 or p <= 0:
            k, T, p = 1, 1.0, 1.0
        n = min(k, o.size) if 0 < k < V else o.size
        top = z[r, o[0]]
        with np.errstate(invalid="ignore", over="ignore"):
            w = np.where(z[r, o[:n]] == top, 1.0, np.exp((z[r, o[:n]] - top) / T) if top < np.inf else 0.0)
        if p < 1:
            before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
            total = w.sum()
            margin[r] = np.min(np.abs(np.cumsum(w)[:-1] - p * total), initial=np.inf) / total
            n = int(np.sum(before < p * total))
        if mp > 0:
            n = min(n, int(np.sum(w[:n] >= mp)))
        keep = np.sort(o[:n])
        back = dict(zip(o[:n].tolist(), w[:n].tolist()))
        wk = np.array([back[i] for i in keep.tolist()])
        cum = np.cumsum(wk)
        at = float(u[r]) * cum[-1]
        j = min(int(np.searchsorted(cum, at, side="right")), n - 1)
        margin[r] = min(margin[r], np.min(np.abs(cum[:-1] - at), initial=np.inf) / cum[-1])
        if np.isin(w, (0.0, 1.0)).all():
            margin[r] = np.inf
        ids[r], logprob[r], n_kept[r] = keep[j], np.log(wk[j] / cum[-1]), n
    return ids, logprob, n_kept, margin
