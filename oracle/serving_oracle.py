"""CPU oracle of the serving operators (test infrastructure): packed prompt attention, loading prompts
into the retained cache, attention of a drafted tree, accepting a drafted path.

Plain fp64 NumPy restatements of the definitions in ``include/tca.h``; no code is shared with the CUDA
library.  The attention functions also return what an error bound needs: for every output the same
sum with |v| in place of v, and for every row the largest sum |q_i k_i| * scale over its visible keys.
"""
from __future__ import annotations

from typing import List, Tuple

import numpy as np

__all__ = ["masked_attention", "packed_attention", "tree_paths", "tree_attention", "load_split", "attention_tolerance"]


def masked_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, visible: np.ndarray, scale: float):
    """softmax(q k^T * scale) v over the visible keys of each row (every row sees at least one); keys that a
    row does not see have no influence whatever they hold.  Returns (o, a, s): a = the same with |v|,
    s[i] = max over visible keys of sum |q_i k_i| * scale."""
    o = np.empty((len(q), v.shape[1]))
    a = np.empty_like(o)
    s = np.empty(len(q))
    for i in range(len(q)):
        j = np.nonzero(visible[i])[0]
        x = (k[j] @ q[i]) * scale
        w = np.exp(x - x.max())
        w /= w.sum()
        o[i], a[i] = w @ v[j], w @ np.abs(v[j])
        s[i] = (np.abs(k[j]) @ np.abs(q[i])).max() * scale
    return o, a, s


def packed_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, starts, scale: float):
    """q [Hq, rows, d], k, v [Hkv, rows, d], starts [n + 1].  Rows of no sequence are NaN in the result."""
    G = q.shape[0] // k.shape[0]
    o = np.full(q.shape, np.nan)
    a = np.full(q.shape, np.nan)
    s = np.full(q.shape[:2], np.nan)
    for lo, hi in zip(starts[:-1], starts[1:]):
        if hi <= lo:
            continue
        tri = np.tril(np.ones((hi - lo, hi - lo), dtype=bool))
        for h in range(q.shape[0]):
            o[h, lo:hi], a[h, lo:hi], s[h, lo:hi] = masked_attention(q[h, lo:hi], k[h // G, lo:hi], v[h // G, lo:hi], tri, scale)
    return o, a, s


def tree_paths(parent: np.ndarray) -> np.ndarray:
    """sees[t, u]: drafted token u lies on t's path to the root (itself included); a parent outside [-1, t) is -1."""
    T = len(parent)
    sees = np.zeros((T, T), dtype=bool)
    for t in range(T):
        p = int(parent[t])
        if 0 <= p < t:
            sees[t] = sees[p]
        sees[t, t] = True
    return sees


def tree_attention(q, k_cache, v_cache, k_draft, v_draft, parent, scale: float):
    """One head: q [T, d] over the unit's cache rows (any order) and the drafted tokens on each path."""
    k, v = np.concatenate([k_cache, k_draft]), np.concatenate([v_cache, v_draft])
    vis = np.concatenate([np.ones((len(q), len(k_cache)), dtype=bool), tree_paths(parent)], axis=1)
    return masked_attention(q, k, v, vis, scale)


def load_split(length: int, window: int, block: int) -> Tuple[int, int]:
    """Rows of a loaded prompt that go to the global region, and to the ring."""
    g = max(0, (length - window) // block) * block
    return g, length - g


def attention_tolerance(o, a, s, d: int, n_keys, dtype: str):
    """Elementwise bound on the kernels' error, from the arithmetic alone.

    A score is a sum of d products accumulated in fp32 (2^-23 per step allows for truncating
    accumulators), scaled once and exponentiated with ex2.approx (2^-22 of its result): a relative
    error of each weight of at most eps_w = 2 * (d + 8) * 2^-23 * s + 2^-21, where s bounds the sum of
    |q_i k_i| * scale.  Numerator and denominator sum n_keys weights in fp32: n_keys * 2^-23 each.
    With bf16 each weight is rounded to bf16 before the second product (half a step, 2^-8 of it,
    numerator only) and the result once more (2^-8 of it); with fp32 the result rounds by 2^-24."""
    n = np.asarray(n_keys, dtype=np.float64)
    eps = 2.0 * (2.0 * (d + 8) * 2.0 ** -23 * s + 2.0 ** -21 + (n + 8) * 2.0 ** -23)
    eps = eps[..., None]
    if dtype == "bf16":
        return a * (eps + 2.0 ** -8) * (1 + eps) + np.abs(o) * 2.0 ** -8 + 2.0 ** -126
    return a * eps * (1 + eps) + np.abs(o) * 2.0 ** -24 + 2.0 ** -126
