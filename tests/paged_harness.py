"""Helpers of the paged-cache tests: caches in a chosen state, views of them on the host, comparison with the oracle."""
from __future__ import annotations

import numpy as np
import torch

import serving_harness as H
from oracle import paged_oracle as P
from paper_2512_09238_b200 import binding as B

ALL = (1 << 31) - 1


def params(batch, hq, hkv, d, dtype, window=ALL):
    return B.make_params(batch, hq, hkv, d, 32, window, sm_scale=H.scale_of(d), dtype=H.DC[dtype])


def make(prm, lens, page, dtype, seed, room=0, spare=2, seen=None, garbage=None, max_pages=None):
    """A cache whose units hold `lens` rows in pages dealt at random, with pages for `room` more.  Everything that is in
    no unit's use holds `garbage` (or finite noise).  seen: position of the next token (default: len)."""
    lens = np.broadcast_to(np.asarray(lens, dtype=np.int64), (prm.batch * prm.n_kv_heads,)).copy()
    need = -(-(lens + room) // page)
    r = np.random.default_rng(seed)
    c = B.PagedCache(prm, int(need.sum()) + spare, page, max_pages or max(1, int(need.max())))
    r.shuffle(c.free)
    c.reserve(lens + room)
    seen = lens if seen is None else np.broadcast_to(np.asarray(seen, dtype=np.int64), lens.shape)
    c.k.copy_(H.randn(seed, tuple(c.k.shape), dtype))
    c.v.copy_(H.randn(seed + 1, tuple(c.v.shape), dtype))
    if garbage is not None:
        rows = [pool_rows(c, u, np.arange(n)) for u, n in enumerate(lens) if n]
        used = torch.from_numpy(np.concatenate(rows) if rows else np.zeros(0, dtype=np.int64)).cuda()
        for t in (c.k, c.v):
            t2 = t.view(-1, prm.head_dim)
            keep = t2[used].clone()
            t2.fill_(garbage)
            t2[used] = keep
    mass = np.exp(r.normal(size=c.n_pages * page)).astype(np.float32)
    c.mass.copy_(torch.from_numpy(mass).view(c.n_pages, page))
    pos = np.full(c.n_pages * page, -7, dtype=np.int32)
    for u, n in enumerate(lens):
        pos[pool_rows(c, u, np.arange(n))] = seen[u] - n + np.arange(n)
    c.pos.copy_(torch.from_numpy(pos).view(c.n_pages, page))
    st = np.zeros((len(lens), B.TCA_PG_STATE_WORDS), dtype=np.int32)
    st[:, B.TCA_PG_LEN], st[:, B.TCA_PG_NEXT] = lens, seen
    c.state.copy_(torch.from_numpy(st))
    return c


def pool_rows(c, u, slots):
    slots = np.asarray(slots, dtype=np.int64)
    return c.table_host[u, slots // c.page_size].astype(np.int64) * c.page_size + slots % c.page_size


def lens_of(c):
    return c.state[:, B.TCA_PG_LEN].cpu().numpy().astype(np.int64)


def snapshot(c):
    """Everything a call can change, on the host, rows flattened."""
    return dict(k=H.f64(c.k).reshape(-1, c.prm.head_dim), v=H.f64(c.v).reshape(-1, c.prm.head_dim), pos=c.pos.cpu().numpy().reshape(-1),
                mass=c.mass.cpu().numpy().reshape(-1), state=c.state.cpu().numpy().copy())


def same(a, b, but=()):
    for name in a:
        if name not in but:
            np.testing.assert_array_equal(a[name], b[name], err_msg=name)


def attend(prm, q, c, n_sink=0, accumulate=False, ws=None, out=None, status=B.TCA_OK):
    o = torch.full_like(q, float("nan")) if out is None else out
    ws = B.alloc_paged_workspace(prm, c, accumulate) if ws is None else ws
    B.tca_attn_paged(prm, q, c, n_sink, accumulate, o, ws)
    assert B.tca_ws_status(ws) == status
    return o


def check(prm, q, c, got, n_sink, dtype, before=None, hidden=None):
    """Compares O (and, with the snapshot before, the masses) with the oracle.  hidden: per unit, slots on bad pages."""
    G, d = prm.n_q_heads // prm.n_kv_heads, prm.head_dim
    s = snapshot(c)
    if before is not None:
        same({k: before[k] for k in ("k", "v", "pos", "state")}, s, ())
    want_mass = None if before is None else before["mass"].astype(np.float64)
    tol_mass = np.zeros(len(s["mass"]))
    qd, o, lens = H.f64(q), H.f64(got), lens_of(c)
    for u in range(prm.batch * prm.n_kv_heads):
        b, h = divmod(u, prm.n_kv_heads)
        slots = P.visible_slots(int(lens[u]), prm.window, n_sink)
        if hidden is not None:
            slots = slots[~np.isin(slots, hidden[u])]
        r = pool_rows(c, u, slots)
        want, a, bound, w = P.paged_attention(qd[b, h * G:(h + 1) * G], s["k"][r], s["v"][r], H.scale_of(d))
        H.check(o[b, h * G:(h + 1) * G], want, P.paged_tolerance(want, a, bound, d, len(r), dtype), f"unit {u}")
        if before is not None:
            tol_mass[r] = P.mass_tolerance(want_mass[r], w, bound, d, len(r))
            want_mass[r] += w
    if before is not None:
        H.check(s["mass"].astype(np.float64), want_mass, tol_mass, "mass")
