"""CPU oracle of the text-generation operators in fp64: rotation and append, attention behind a shared prefix, sampling.

Test infrastructure only.  Written from the definitions in include/freeride.h, one token and one head at a time.
"""
import numpy as np


def rotate(x, cos, sin, rotary_dim, pairs):
    """x [heads, head_dim] fp64; cos, sin [rotary_dim / 2]."""
    y = np.array(x, dtype=np.float64)
    half = rotary_dim // 2
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
        y[:, a] = x[:, a] * cos[i] - x[:, b] * sin[i]
        y[:, b] = x[:, b] * cos[i] + x[:, a] * sin[i]
    return y


def visible(prefix_len, own_len, t, i):
    """Keys that token i of t sees: the prefix and the first own_len - t + 1 + i own ones."""
    return prefix_len + max(0, own_len - t + 1 + i)


def attend_row(q, k, v, scale):
    """q [D]; k, v [n, D], all fp64 -> (out [D], lse, sum p |v| / sum p, largest sum |q_i k_i|)."""
    if len(k) == 0:
        return np.zeros(len(q)), -np.inf, np.zeros(len(q)), 0.0
    with np.errstate(over="ignore", invalid="ignore"):
        x = scale * (k @ q)
        m = x.max()
        e = np.exp(x - m)
        total = e.sum()
        return (e @ v) / total, m + np.log(total), (e @ np.abs(v)) / total, scale * (np.abs(k) @ np.abs(q)).max()


def weights(logits, temperature):
    """fp64 weights relative to the largest logit; None for a row without any."""
    x = np.where(np.isnan(logits), -np.inf, np.asarray(logits, dtype=np.float64))
    top = x.max()
    if top == -np.inf:
        return None, x
    with np.errstate(over="ignore", invalid="ignore"):
        w = np.where(x == top, 1.0, np.where(x == -np.inf, 0.0, np.exp((x - top) / temperature)))
    return w, x


def kept(logits, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """Indices kept, ascending, and the weights."""
    w, x = weights(logits, temperature)
    order = np.argsort(-x, kind="stable")
    if 0 < top_k < len(order):
        order = order[:top_k]
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[order])[:-1]])
        n = int((before < top_p * w[order].sum()).sum())
        order = order[:max(1, n)]
    order = order[~(w[order] < min(min_p, 1.0))]
    return np.sort(order), w


def sample(logits, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    x = np.where(np.isnan(logits), -np.inf, np.asarray(logits, dtype=np.float64))
    if x.max() == -np.inf:
        return -1
    if not temperature > 0:
        return int(np.argmax(x))
    index, w = kept(logits, temperature, top_k, top_p, min_p)
    run = np.cumsum(w[index])
    return int(index[min(np.searchsorted(run, uniform * run[-1], side="right"), len(index) - 1)])
