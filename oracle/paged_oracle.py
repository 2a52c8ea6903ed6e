"""CPU oracle of the paged-cache operators (test infrastructure): prompt attention with a sliding window and sinks,
attention of one token over a paged cache with the weights it gives, eviction by accumulated weight.

Plain fp64 NumPy restatements of the definitions in ``include/tca.h``; no code is shared with the CUDA library.
"""
from __future__ import annotations

import numpy as np

from oracle.serving_oracle import masked_attention

__all__ = ["window_mask", "window_attention", "visible_slots", "paged_attention", "evict", "paged_tolerance", "mass_tolerance"]


def window_mask(n: int, window: int, n_sink: int) -> np.ndarray:
    """sees[i, j]: row i of a prompt of n rows attends to row j."""
    i, j = np.arange(n)[:, None], np.arange(n)[None, :]
    return (j <= i) & ((i - j < window) | (j < n_sink))


def window_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, starts, window: int, n_sink: int, scale: float):
    """q [Hq, rows, d], k, v [Hkv, rows, d], starts [n + 1].  Rows of no sequence are NaN in the result (o, a, s as in
    masked_attention)."""
    G = q.shape[0] // k.shape[0]
    o, a, s = np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.full(q.shape[:2], np.nan)
    for lo, hi in zip(starts[:-1], starts[1:]):
        if hi <= lo:
            continue
        sees = window_mask(hi - lo, window, n_sink)
        for h in range(q.shape[0]):
            o[h, lo:hi], a[h, lo:hi], s[h, lo:hi] = masked_attention(q[h, lo:hi], k[h // G, lo:hi], v[h // G, lo:hi], sees, scale)
    return o, a, s


def visible_slots(length: int, window: int, n_sink: int) -> np.ndarray:
    j = np.arange(length)
    return j[(j >= length - window) | (j < n_sink)]


def paged_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """q [G, d] over a unit's visible rows k, v [n, d]: (o, a, s, w), w [n] the mean over the heads of the softmax weights;
    zeros where nothing is visible."""
    if len(k) == 0:
        return np.zeros(q.shape), np.zeros(q.shape), np.zeros(len(q)), np.zeros(0)
    o, a, s = masked_attention(q, k, v, np.ones((len(q), len(k)), dtype=bool), scale)
    x = q @ k.T * scale
    w = np.exp(x - x.max(1, keepdims=True))
    return o, a, s, (w / w.sum(1, keepdims=True)).mean(0)


def evict(mass: np.ndarray, pos: np.ndarray, budget: int, n_sink: int, n_recent: int):
    """Which slot's row every slot below the budget holds afterwards ([budget] source slots), or None if the unit stays
    as it was because its safe rows are too many.  A unit within its budget keeps all rows where they are."""
    n = len(mass)
    if n <= budget:
        return np.arange(n)
    safe = [j for j in range(n) if j < n_sink or int(pos[j]) > int(pos.max()) - n_recent]
    if len(safe) > budget:
        return None
    rest = [j for j in range(n) if j not in set(safe)]
    weight = {j: np.inf if np.isnan(mass[j]) else float(mass[j]) for j in rest}
    rest.sort(key=lambda j: (not np.isnan(mass[j]), -weight[j], j))
    kept = set(safe) | set(rest[:budget - len(safe)])
    source = np.arange(budget)
    holes = [j for j in range(budget) if j not in kept]
    late = [j for j in range(budget, n) if j in kept]
    source[holes] = late
    return source


def paged_tolerance(o, a, s, d: int, n_keys: int, dtype: str):
    """serving_oracle.attention_tolerance for one unit: the same arithmetic, and the merges of the warps' and shares'
    states (at most 4 + log2 steps of a warp reduction + one per share, each a product and a sum in fp32): 200 more
    roundings of 2^-23."""
    eps = (2.0 * (2.0 * (d + 8) * 2.0 ** -23 * s + 2.0 ** -21 + (n_keys + 200) * 2.0 ** -23))[..., None]
    if dtype == "bf16":
        return a * (eps + 2.0 ** -8) * (1 + eps) + np.abs(o) * 2.0 ** -8 + 2.0 ** -126
    return a * eps * (1 + eps) + np.abs(o) * 2.0 ** -24 + 2.0 ** -126


def mass_tolerance(before, added, s: float, d: int, n_keys: int):
    """A weight is exp2(x - lse): x carries the error of a score (paged_tolerance), lse that of the scores and of a sum
    of n_keys terms, both are rounded once more (2^-24 of at most s log2(e) + log2(n)); then the G weights are added and
    the sum is rounded into the mass (2^-24 of it)."""
    s = float(np.max(s, initial=0.0))
    eps = 2.0 * (2.0 * (d + 16) * 2.0 ** -23 * (s + np.log2(n_keys + 1)) + 2.0 ** -20 + (n_keys + 200) * 2.0 ** -23)
    return added * eps * (1 + eps) + np.abs(before + added) * 2.0 ** -23 + 2.0 ** -126
