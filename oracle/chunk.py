"""Several new tokens of a sequence at once: rotation, attention of the rows, probabilities and verification of drafts, in 64 bits (oracle side).

TEST INFRASTRUCTURE ONLY; shares no code with the HIP library.
"""
import math

import numpy as np


def rotate(x, positions, inv_freq, interleaved):
    """x [rows][heads][d]; pair j of the first 2 len(inv_freq) elements turned by positions[row] * inv_freq[j]."""
    y = np.array(x, dtype=np.float64)
    n = len(inv_freq)
    for j in range(n):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + n)
        angle = np.asarray(positions, dtype=np.float64)[:, None] * inv_freq[j]
        u, v = np.array(y[..., a]), np.array(y[..., b])
        y[..., a], y[..., b] = u * np.cos(angle) - v * np.sin(angle), u * np.sin(angle) + v * np.cos(angle)
    return y


def sees(p, n_keys, window, prefix):
    """Which of keys 0 .. n_keys - 1 a row at position p sees."""
    i = np.arange(n_keys)
    recent = (i <= p) & ((i > p - window) if window else True)
    return recent | (i < prefix)


def attend(q, K, V, p, scale=0.0, cap=0.0, window=0, slope=0.0, prefix=0):
    """One row: q [d], K and V [n][d] (all of the sequence's tokens), position p.  -> (out [d], weighted mean of |v| [d], largest scale * sum |q k|)"""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    scale = scale or 1.0 / math.sqrt(len(q))
    seen = sees(p, len(K), window, prefix)
    if not seen.any():
        return np.zeros(len(q)), np.zeros(len(q)), 0.0
    K, V, i = K[seen], V[seen], np.arange(len(seen))[seen]
    s = scale * (K @ q)
    if cap:
        s = cap * np.tanh(s / cap)
    s = s - slope * np.abs(p - i)
    top = s.max()
    if top == -math.inf:
        return np.zeros(len(q)), np.zeros(len(q)), 0.0
    w = np.exp(s - top)
    there = w > 0
    w, V = w[there], V[there]
    return w @ V / w.sum(), w @ np.abs(V) / w.sum(), scale * (np.abs(K) @ np.abs(q)).max()


def probs(logits, t):
    """One row."""
    x = np.asarray(logits, dtype=np.float64)
    if x.max() == -math.inf:
        return np.zeros(len(x))
    if t == 0:
        out = np.zeros(len(x))
        out[int(np.argmax(x))] = 1
        return out
    e = np.exp((x - x.max()) / t)
    return e / e.sum()


def verify(target, draft_probs, drafts, uniforms):
    """One sequence: target [n + 1][V], draft_probs [n][V] or None, drafts [n], uniforms [n + 1], fp32.  -> (tokens [n + 1], accepted)"""
    n, V = len(drafts), target.shape[1]
    a = 0
    while a < n and 0 <= drafts[a] < V:
        q = np.float32(1) if draft_probs is None else draft_probs[a, drafts[a]]
        if not np.float32(uniforms[a]) * q < target[a, drafts[a]]:
            break
        a += 1

    def clean(w):
        return np.where(np.isfinite(w) & (w > 0), w, 0.0)

    w = np.asarray(target[a], dtype=np.float64)
    all_of_it = clean(w)
    if a < n:
        off = np.zeros(V)
        if draft_probs is not None:
            off = np.asarray(draft_probs[a], dtype=np.float64)
        elif 0 <= drafts[a] < V:
            off[drafts[a]] = np.inf
        with np.errstate(invalid="ignore"):
            w = clean(w - off)
        if not w.any():
            w = all_of_it
    else:
        w = all_of_it
    token = -1
    if w.any():
        upto = np.cumsum(w)
        token = int(np.argmax(upto > float(uniforms[n]) * upto[-1]))
    return [*[int(x) for x in drafts[:a]], token, *[-1] * (n - a)], a
