"""The operators around a layer that serves k experts per token, in plain float64 numpy, one token after the other: what the
tests compare the library with.  Shares no code with it."""
from __future__ import annotations

import numpy as np

E4M3 = np.array([(1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6 for e in range(16) for m in range(8)][:127])   # 0 .. 448


def e4m3_values(q: np.ndarray) -> np.ndarray:
    """Bytes -> the numbers they stand for (no NaN among them)."""
    assert not ((q & 127) == 127).any()
    return np.where(q & 128, -1.0, 1.0) * E4M3[q & 127]


def scale_exponent(amax: np.ndarray) -> np.ndarray:
    """Smallest e in [-126, 127] with amax <= 448 * 2^e."""
    e = np.full(amax.shape, -126)
    for _ in range(254):
        up = amax > 448 * 2.0 ** e.astype(np.float64)
        if not up.any():
            break
        e = np.minimum(e + up, 127)
    return e


def to_blocks(v: np.ndarray):
    """float64 [..., n] -> (e4m3 values in units of the scale, exponents [..., n / 32]): nearest, ties to the even one."""
    b = v.reshape(*v.shape[:-1], -1, 32)
    e = scale_exponent(np.abs(b).max(-1))
    u = np.abs(b) / 2.0 ** e[..., None].astype(np.float64)
    hi = np.searchsorted(E4M3, u).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = u - E4M3[lo], E4M3[hi] - u
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (np.sign(b) * E4M3[pick]).reshape(v.shape), e


def from_blocks(q: np.ndarray, e: np.ndarray) -> np.ndarray:
    return (q.reshape(*q.shape[:-1], -1, 32) * 2.0 ** e[..., None].astype(np.float64)).reshape(q.shape)


def add_norm(x, res, w, eps):
    h = x if res is None else x + res
    return h, h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * w


def choose(scores, biased, k, groups, kept, best, renorm, scale):
    """One token: ids (-1: none) and weights of its k choices, by plain sorting."""
    E = len(scores)
    per = E // groups
    ranks = []
    for g in range(groups):
        top = sorted((v for v in biased[g * per:(g + 1) * per] if v > -np.inf), reverse=True)[:best]
        ranks.append(sum(top) if top else -np.inf)
    keep = [g for g in sorted(range(groups), key=lambda g: (-ranks[g], g))[:kept] if ranks[g] > -np.inf]
    have = [e for e in range(E) if e // per in keep and biased[e] > -np.inf]
    ids = sorted(have, key=lambda e: (-biased[e], e))[:k]
    w = np.array([scores[e] for e in ids])
    if renorm and len(ids):
        w = w / w.sum()
    return ids + [-1] * (k - len(ids)), list(w * scale) + [0.0] * (k - len(ids))


def route(x, Wr, e2s, k, sigmoid=False, bias=None, groups=1, kept=1, best=1, renorm=True, scale=1.0):
    """float64 x [T, d] -> dict of orig_expert, orig_gate, slot, gate [T, k] and xnorm [T]."""
    z = x @ Wr.T
    s = 1 / (1 + np.exp(-z)) if sigmoid else np.exp(z - z.max(1, keepdims=True))
    if not sigmoid:
        s /= s.sum(1, keepdims=True)
    out = {n: [] for n in ("orig_expert", "orig_gate", "slot", "gate")}
    for t in range(len(x)):
        b = s[t] + (0 if bias is None else bias)
        i, w = choose(s[t], b, k, groups, kept, best, renorm, scale)
        out["orig_expert"].append(i)
        out["orig_gate"].append(w)
        i, w = choose(s[t], np.where(e2s >= 0, b, -np.inf), k, groups, kept, best, renorm, scale)
        out["slot"].append([-1 if e < 0 else e2s[e] for e in i])
        out["gate"].append(w)
    return {n: np.array(v).reshape(len(x), k) for n, v in out.items()} | {"xnorm": np.sqrt((x * x).sum(1))}


def sort_pairs(slot, K):
    """slot [n] -> perm (served pairs in slot order), inverse (-1: not served), offsets [K + 1]."""
    perm = [i for s in range(K) for i in np.flatnonzero(slot == s)]
    inv = np.full(len(slot), -1)
    inv[perm] = np.arange(len(perm))
    return np.array(perm, int), inv, np.array([(np.asarray(slot)[(slot >= 0) & (slot < K)] < s).sum() for s in range(K + 1)])


def expert_ffn(x, w1, w2):
    """Rows of one slot on weights already rounded to blocks: (y, hidden before its rounding)."""
    h = np.maximum(x @ w1, 0)
    return from_blocks(*to_blocks(h)) @ w2, h


def round_columns(w):
    """A weight matrix [R, N] rounded to blocks of 32 along the reduction, the last block filled with zeros."""
    r = w.shape[0]
    pad = np.zeros((-r % 32, w.shape[1]))
    return from_blocks(*to_blocks(np.concatenate([w, pad]).T)).T[:r]
