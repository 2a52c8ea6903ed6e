"""Helpers of the serving-operator tests: seeded inputs, caches in a chosen state, comparison with the oracle
under the bound the arithmetic allows."""
from __future__ import annotations

import math

import numpy as np
import torch

from oracle import serving_oracle as S
from paper_2512_09238_b200 import binding as B

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DC = {"bf16": B.TCA_BF16, "f32": B.TCA_F32}


def scale_of(d):
    return float(np.float32(1.0 / math.sqrt(d)))


def params(batch, hq, hkv, d, dtype, block=32, window=64, flags=0):
    return B.make_params(batch, hq, hkv, d, block, window, sm_scale=scale_of(d), dtype=DC[dtype], flags=flags)


def randn(seed, shape, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(DT[dtype]).cuda()


def f64(t):
    return t.detach().cpu().double().numpy()


def packed_buffer(seed, heads, rows, d, dtype, layout):
    """[heads, rows, d]: contiguous ("heads"), a view of [rows, heads, d] ("tokens"), or of a wider token-major
    buffer as a fused projection leaves it ("fused"), or rows that are aligned to 16 bytes only ("odd")."""
    if layout == "heads":
        return randn(seed, (heads, rows, d), dtype)
    if layout == "tokens":
        return randn(seed, (rows, heads, d), dtype).transpose(0, 1)
    if layout == "odd":     # rows 16 bytes longer than needed, starting 16 bytes into the buffer
        pad = 16 // DT[dtype].itemsize
        return randn(seed, (heads, rows, d + pad), dtype)[:, :, pad:]
    return randn(seed, (rows, heads + 3, d), dtype)[:, 2:2 + heads].transpose(0, 1)


def run_packed(prm, q, k, v, starts, out=None, ws=None):
    o = torch.full_like(q, float("nan")) if out is None else out
    ws = B.alloc_workspace(prm, max(1, q.shape[1]), B.TCA_OP_PACKED) if ws is None else ws
    st = torch.tensor(np.asarray(starts), dtype=torch.int64, device="cuda")
    B.tca_attn_packed(prm, q, k, v, q.shape[1], st, o, ws)
    assert B.tca_ws_status(ws) == B.TCA_OK
    return o


def check(got, want, tol, what=""):
    """|got - want| <= tol elementwise; NaN in `want` means: must be left as the NaN it was."""
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: rows written that are nobody's, or NaN where a value belongs"
    bad = np.abs(got - want) > tol
    assert not np.any(bad), f"{what}: {np.sum(bad)} of {bad.size} outside the bound, worst ratio {np.nanmax(np.abs(got - want) / tol):.3g}"


def make_cache(prm, n_global, n_tail, head, seq_len, dtype, seed, t_keep=None, extra_cap=0, tail_cap=None):
    """A cache whose units hold the given numbers of rows; unused rows hold finite garbage."""
    U = prm.batch * prm.n_kv_heads
    as64 = lambda x: np.broadcast_to(np.asarray(x, dtype=np.int64), (U,)).copy()  # noqa: E731
    n_global, n_tail, head, seq_len = as64(n_global), as64(n_tail), as64(head), as64(seq_len)
    tk = as64(4 if t_keep is None else t_keep)
    c = B.Cache(prm, n_global + extra_cap, tail_cap or prm.window + prm.block, tk, init=False)
    for name, x in (("n_global", n_global), ("n_tail", n_tail), ("tail_head", head), ("seq_len", seq_len)):
        getattr(c, name)[:] = x
    B.tca_cache_init(prm, c)
    c.k.copy_(randn(seed, tuple(c.k.shape), dtype))
    c.v.copy_(randn(seed + 1, tuple(c.v.shape), dtype))
    pos = np.full(c.rows_total, -1, dtype=np.int32)
    for u in range(U):
        rows = c.unit_rows(u)
        pos[rows] = np.concatenate([np.arange(n_global[u]), seq_len[u] - n_tail[u] + np.arange(n_tail[u])])
    c.pos.copy_(torch.from_numpy(pos))
    return c


def clone_cache(prm, c):
    d = B.Cache(prm, c.global_cap, c.tail_cap, c.t_keep, init=False)
    for name in ("n_global", "n_tail", "tail_head", "seq_len"):
        getattr(d, name)[:] = getattr(c, name)
    B.tca_cache_init(prm, d)
    for name in ("k", "v", "pos", "state"):
        getattr(d, name).copy_(getattr(c, name))
    return d


def mirror_equals_device(c):
    st = c.state.cpu().numpy().reshape(-1, B.TCA_STATE_WORDS)
    for i, name in enumerate(("seg_start", "global_cap", "n_global", "tail_head", "n_tail", "seq_len", "t_keep")):
        np.testing.assert_array_equal(st[:, i], getattr(c, name), err_msg=name)


def chain(T):
    return np.arange(-1, T - 1, dtype=np.int32)


def bush(T, seed):
    r = np.random.default_rng(seed)
    return np.array([-1 if t < 3 else int(r.integers(-1, t)) for t in range(T)], dtype=np.int32)


def run_tree(prm, q, kd, vd, parent, cache, n_live=None, out=None, ws=None):
    T = q.shape[2]
    o = torch.full_like(q, float("nan")) if out is None else out
    ws = B.alloc_tree_workspace(prm, T) if ws is None else ws
    nl = None if n_live is None else torch.tensor(np.asarray(n_live, dtype=np.int32), device="cuda")
    B.tca_attn_tree(prm, q, kd, vd, T, torch.from_numpy(np.ascontiguousarray(parent)).cuda(), nl, cache, o, ws)
    assert B.tca_ws_status(ws) == B.TCA_OK
    return o


def check_tree_rows(prm, q, kd, vd, parent, cache, got, dtype):
    """check_tree for a cache too large to copy: only the rows in use come to the host."""
    class Rows:
        def __init__(self, x):
            self.x = x

        def __getitem__(self, rows):
            return f64(self.x[torch.from_numpy(rows).cuda()])

    check_tree(prm, q, kd, vd, parent, cache, got, dtype, kv=(Rows(cache.k), Rows(cache.v)))


def check_tree(prm, q, kd, vd, parent, cache, got, dtype, n_live=None, heads=None, kv=None):
    """Compares every (or the given) query head's rows with the oracle."""
    G, T = prm.n_q_heads // prm.n_kv_heads, q.shape[2]
    k, v = kv or (f64(cache.k), f64(cache.v))
    qd, kdd, vdd, o = f64(q), f64(kd), f64(vd), f64(got)
    for s in range(prm.batch):
        n = T if n_live is None else int(n_live[s])
        for h in range(prm.n_q_heads):
            if heads is not None and h not in heads:
                continue
            u = s * prm.n_kv_heads + h // G
            rows = cache.unit_rows(u)
            want, a, ss = S.tree_attention(qd[s, h], k[rows], v[rows], kdd[s, h // G], vdd[s, h // G], parent[s], scale_of(prm.head_dim))
            tol = S.attention_tolerance(want, a, ss, prm.head_dim, np.full(T, len(rows) + T), dtype)
            want[n:], tol[n:] = np.nan, 1.0
            check(o[s, h], want, tol, f"sequence {s} head {h}")
