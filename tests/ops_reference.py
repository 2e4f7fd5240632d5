"""Plain 64-bit forms of the operators that take no model, in numpy: 4-bit products, the draw of a word, distillation."""
import numpy as np


def unpack_codes(codes, H):
    c = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1)
    return c[:, :H].astype(np.int64)


def q4_weights(codes, H, group, scales, zeros):
    """float64 [V, H] weights; scales [groups, V] as float64."""
    of = np.arange(H) // group
    z = np.full(scales.shape, 8.0) if zeros is None else zeros.astype(np.float64)
    return (unpack_codes(codes, H) - z.T[:, of]) * scales.T.astype(np.float64)[:, of]


def sample_row(z, u, T=1.0, k=0, p=1.0, m=0.0):
    """(word, logprob, its weight relative to the row's maximum) of one row of logits."""
    z = np.asarray(z, np.float64)
    V = len(z)
    bad = (-1, np.nan, 1.0)
    if np.isnan(z).any() or not z.max() > -np.inf or not (0 <= T < np.inf) or not (0 <= u < 1) or np.isnan(p) or np.isnan(m):
        return bad
    order = np.argsort(-z, kind="stable")
    if T == 0:
        return int(order[0]), 0.0, 1.0
    if z.max() == np.inf:
        w = (z == np.inf).astype(np.float64)
    else:
        w = np.exp((z - z.max()) / T)
    kept = order[:k] if 0 < k < V else order
    if p < 1:
        upto = np.cumsum(w[kept])
        kept = kept[:max(1, int(np.searchsorted(upto, p * upto[-1], side="left")) + 1)]
    kept = kept[w[kept] >= min(m, 1.0)] if m > 0 else kept
    mass = np.zeros(V)
    mass[kept] = w[kept]
    upto = np.cumsum(mass)
    word = int(np.searchsorted(upto, u * upto[-1], side="right"))
    return word, float(np.log(mass[word] / upto[-1])), float(w[word])


def distill_row(z, words, logits, label, T, a, V=None):
    """(loss, gradient, max |log p|, |log q| that counts) of one row."""
    z = np.asarray(z, np.float64)
    V = len(z)
    words, t = np.asarray(words), np.asarray(logits, np.float64)
    nan = (np.nan, np.full(V, np.nan), 0.0)
    if ((words < -1) | (words >= V)).any() or not -1 <= label < V:
        return nan
    words, t = words[words >= 0], t[words >= 0]
    if np.isnan(t).any() or (t == np.inf).any():
        return nan
    soft = len(t) > 0 and t.max() > -np.inf and a < 1
    hard = label >= 0 and a > 0
    if not soft and not hard:
        return 0.0, np.zeros(V), 0.0
    if np.isnan(z).any() or not -np.inf < z.max() < np.inf:
        return nan
    loss, grad, far = 0.0, np.zeros(V), 0.0
    with np.errstate(divide="ignore"):
        if soft:
            y = (z - z.max()) / T
            log_p = y - np.log(np.exp(y).sum())
            s = (t - t.max()) / T
            log_q = s - np.log(np.exp(s).sum())
            q = np.exp(log_q)
            on = q > 0
            loss += (1 - a) * T * T * (q[on] * (log_q[on] - log_p[words[on]])).sum()
            grad += (1 - a) * T * np.exp(log_p)
            np.subtract.at(grad, words, (1 - a) * T * q)
            far = max(np.abs(log_q[on]).max(), np.abs(log_p[words[on]]).max())
        if hard:
            y = z - z.max()
            log_p = y - np.log(np.exp(y).sum())
            loss -= a * log_p[label]
            grad += a * np.exp(log_p)
            grad[label] -= a
            far = max(far, abs(log_p[label]))
    return loss, grad, far
