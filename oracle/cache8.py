"""CPU oracle of a cache held in 8 bits, in fp64: codes and scales, the append, which keys a token sees, copies of pages.

Test infrastructure only.  Written from the definitions in include/freeride.h; attention itself is oracle/generation.py's.
"""
import numpy as np

from .generation import rotate

RANGE = {"bf16": (10, 246), "f16": (112, 134)}


def _value(code):
    e, m = code >> 3 & 15, code & 7
    if e == 15 and m == 7:
        return np.nan
    x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    return -x if code & 128 else x


VALUES = np.array([_value(c) for c in range(256)])
_MIDDLE = (VALUES[:126] + VALUES[1:127]) / 2            # between neighbouring codes 0 .. 126 (448)


def encode(y):
    """Codes nearest to y, ties to the even code, at most 448; NaN and infinities give NaN (0x7f; its sign is not checked)."""
    y = np.asarray(y, dtype=np.float64)
    a = np.abs(np.where(np.isfinite(y), y, 0))
    i = np.searchsorted(_MIDDLE, a, side="left")
    tie = (i < 126) & (a == _MIDDLE[np.minimum(i, 125)])
    i = np.where(tie & (i % 2 == 1), i + 1, i)
    code = np.where(np.isfinite(y), i, 127)
    return (code + np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def scale_of(byte, dtype):
    return 2.0 ** (np.clip(np.asarray(byte, dtype=np.int64), *RANGE[dtype]) - 127)


def need(x, dtype):
    """The least scale byte whose 448 2^(s - 127) is the largest finite magnitude of x or more."""
    lo, hi = RANGE[dtype]
    x = x[np.isfinite(x)]
    top = np.abs(x).max() if x.size else 0.0
    for s in range(lo, hi):
        if 448 * 2.0 ** (s - 127) >= top:
            return s
    return hi


def numbers(codes, scale, block, dtype):
    """Numbers [pages, heads, slots, dim] that codes and scale bytes [pages, heads, slots / block] stand for."""
    return VALUES[codes] * np.repeat(scale_of(scale, dtype), block, axis=2)[..., None]


def append(ck, cv, sk, sv, k, v, slot, block, dtype, cos=None, sin=None, rotary_dim=0, pairs=False):
    """In place: codes [pages, heads, page, dim] and scale bytes; k, v [tokens, heads, dim] fp64; cos, sin [tokens, rotary_dim / 2] fp64."""
    pages, heads, page, _ = ck.shape
    x = np.stack([rotate(k[t], cos[t], sin[t], rotary_dim, pairs) if rotary_dim else k[t] for t in range(len(k))]) if len(k) else k
    blocks = {}
    for t, s in enumerate(slot):
        if 0 <= s < pages * page:
            blocks.setdefault(int(s) // block, []).append(t)
    for b, tokens in blocks.items():
        p, first = b * block // page, b * block % page
        own = [int(slot[t]) % page for t in tokens]
        for codes, scale, new in ((ck, sk, x), (cv, sv, v)):
            for h in range(heads):
                s = need(new[tokens, h], dtype)
                old = int(np.clip(scale[p, h, first // block], *RANGE[dtype]))
                if first not in own:
                    s = max(s, old)
                    if s > old:
                        for o in range(first, first + block):
                            if o not in own:
                                codes[p, h, o] = encode(VALUES[codes[p, h, o]] * 2.0 ** (old - s))
                for t, o in zip(tokens, own):
                    codes[p, h, o] = encode(new[t, h] * 2.0 ** (127 - s))
                scale[p, h, first // block] = s


def seen(length, t, i, window, sinks):
    """Keys that token i of t sees, ascending."""
    n = max(0, length - t + 1 + i)
    j = np.arange(n)
    return j[(j >= n - window) | (j < sinks)] if window else j


def copies(source, target, n_pages):
    """Which pairs are carried out."""
    inside = lambda i: 0 <= source[i] < n_pages and 0 <= target[i] < n_pages and source[i] != target[i]
    real = [i for i in range(len(source)) if inside(i)]
    return [i in real and not any(target[j] == target[i] and j > i or target[j] == source[i] and j != i for j in real) for i in range(len(source))]
