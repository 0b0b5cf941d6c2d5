"""Float64 definitions of the probabilities of logits and of the verification of drafted tokens (numpy, plain loops)."""
import numpy as np


def probs(logits, temperature=None):
    """logits [rows][vocab] (float32 values) -> float64 probabilities."""
    x = np.asarray(logits, dtype=np.float64)
    out = np.zeros(x.shape)
    for r in range(x.shape[0]):
        t = 1.0 if temperature is None else float(temperature[r])
        if np.isnan(x[r]).any() or (t > 0 and np.isposinf(x[r]).any()):
            out[r] = np.nan
        elif np.isneginf(x[r]).all():
            out[r] = 0
        elif t > 0:
            d = x[r] - x[r].max()
            w = np.where(np.isneginf(d), 0.0, np.exp(np.where(np.isneginf(d), 0.0, d) / t))
            out[r] = w / w.sum()
        else:
            out[r, int(np.argmax(x[r]))] = 1
    return out


def draw(r, u):
    """The lowest index whose running sum exceeds u times the sum; -1 where there is nothing."""
    r = np.where(r > 0, r, 0.0)
    c = np.cumsum(r)
    if not c[-1] > 0:
        return -1
    return min(int(np.sum(c <= u * c[-1])), int(np.nonzero(r)[0][-1]))


def verify(p, q, drafts, uniforms, counts=None):
    """-> (tokens [batch][n + 1], accepted [batch]); rows of padding are None."""
    p, u = np.asarray(p, dtype=np.float64), np.asarray(uniforms, dtype=np.float64)
    q = None if q is None else np.asarray(q, dtype=np.float64)
    batch, n, vocab = p.shape[0], p.shape[1] - 1, p.shape[2]
    tokens, accepted = [], []
    for b in range(batch):
        count = n if counts is None else int(counts[b])
        if count < 0:
            tokens.append(None), accepted.append(None)
            continue
        count, kept, row = min(count, n), [], None
        for i in range(count):
            t = int(drafts[b][i])
            inside = 0 <= t < vocab
            if inside and u[b, i] * (1.0 if q is None else q[b, i, t]) < p[b, i, t]:
                kept.append(t)
                continue
            other = np.zeros(vocab)
            if q is not None:
                other = q[b, i]
            elif inside:
                other[t] = np.inf                     # nothing of a certain draft is left
            row = np.where(p[b, i] - other > 0, p[b, i] - other, 0.0)
            if not row.sum() > 0:
                row = p[b, i]
            break
        if row is None:
            row = p[b, count]
        accepted.append(len(kept))
        tokens.append(kept + [draw(row, u[b, n])] + [-1] * (n - len(kept)))
    return tokens, accepted
