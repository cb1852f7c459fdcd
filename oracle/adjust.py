"""64-bit implementation of the adjusted logits and their gradient, token by token in numpy, from the definition.

Rows are float64 arrays that hold the exact bf16 or fp32 values; a setting is None where nobody sets it.
"""
import numpy as np


def _history(V, hist, length):
    ids = hist[:length]
    return ids[(ids >= 0) & (ids < V)]


def _allowed(V, words):
    v = np.arange(V)
    return (words.astype(np.uint32)[v // 32] >> (v % 32).astype(np.uint32)) & 1 == 1


def adjust(z, hist=None, hist_len=None, n_prompt=None, repetition=None, presence=None, frequency=None,
           bias=None, mask=None, mask_row=None):
    """bias: for each row a dict from token to value.  hist [B][L]; mask [n][words]."""
    B, V = z.shape
    out = z.copy()
    for b in range(B):
        if hist is not None:
            n = hist.shape[1] if hist_len is None else int(hist_len[b])
            first = 0 if n_prompt is None else max(0, int(n_prompt[b]))
            r = 1.0 if repetition is None else float(repetition[b])
            for v in set(_history(V, hist[b], n).tolist()):
                out[b, v] = z[b, v] / r if z[b, v] > 0 else z[b, v] * r
            made = hist[b][:n][first:]
            for v in made[(made >= 0) & (made < V)].tolist():
                out[b, v] -= 0.0 if frequency is None else float(frequency[b])
            for v in set(made[(made >= 0) & (made < V)].tolist()):
                out[b, v] -= 0.0 if presence is None else float(presence[b])
        if bias is not None:
            for v, x in bias[b].items():
                out[b, v] = -np.inf if x == -np.inf else out[b, v] + x
        if mask is not None:
            m = b if mask_row is None else int(mask_row[b])
            if m >= 0:
                out[b, ~_allowed(V, mask[m])] = -np.inf
    return out


def grad(z, dout, hist=None, hist_len=None, repetition=None, mask=None, mask_row=None):
    B, V = z.shape
    d = dout.copy()
    for b in range(B):
        if hist is not None and repetition is not None:
            n = hist.shape[1] if hist_len is None else int(hist_len[b])
            r = float(repetition[b])
            for v in set(_history(V, hist[b], n).tolist()):
                d[b, v] = dout[b, v] / r if z[b, v] > 0 else dout[b, v] * r
        if mask is not None:
            m = b if mask_row is None else int(mask_row[b])
            if m >= 0:
                d[b, ~_allowed(V, mask[m])] = 0.0
    return d
