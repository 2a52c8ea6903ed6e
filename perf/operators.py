"""Workloads of the serving operators: packed prompt attention, loading prompts into the retained
cache, attention of a drafted tree over that cache, and accepting a drafted path.

``listed()`` and ``draw()`` name cases, ``prepare()`` makes their inputs, ``run()`` is one call of
the operator: in its plain form (elementary torch operations, 32 bits or more, rounded once at the
end) or, where ``own`` is set, through the library.  ``exact()`` is the operator's definition in
64 bits.  ``work()`` states the bytes and floating-point operations a pass cannot do without.

Definitions (positions 0-based, scale = 1/sqrt(head_dim) as a float32):
  packed  sequence s owns rows [start[s], start[s+1]); row i of it attends to rows j <= i of it.
  load    sequence s of length len goes to cache sequence slot[s]: with m = max(0, (len - window) //
          block), rows [0, m*block) to the unit's global region, the rest to its ring from slot 0.
  tree    query (head, t) attends to every row of its unit's cache and to the drafted tokens on its
          own path to the root (parent[t] < t, -1 at the root), itself included.
  accept  the drafted tokens path[0..n) are appended one after another; whenever the ring then holds
          window + block tokens, its oldest block is scored with that token's queries, the t_keep best
          rows move to the end of the global region in order and the rest are dropped.
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F32 = "bf16", "f32"
TREE_MAX = 128          # drafted tokens per sequence
STATE_WORDS = 8


# ------------------------------------------------------------------ cases
def listed():
    return [
        # three short prompts that arrive together (a tool call, a greeting, a one-token probe): latency
        dict(name="packed short bf16", op="packed", dtype=BF16, hq=32, hkv=8, d=128, n_seq=3, max_len=40,
             layout="heads", lens=1),
        # a batch of chat turns of very different lengths, token-major as a fused projection writes it
        dict(name="packed chat bf16", op="packed", dtype=BF16, hq=32, hkv=8, d=128, n_seq=24, max_len=1024,
             layout="tokens", lens=2),
        # long documents: the prompts the window makes dense, and a few times longer ones
        dict(name="packed long bf16", op="packed", dtype=BF16, hq=32, hkv=8, d=128, n_seq=3, max_len=8192,
             layout="heads", lens=3),
        # the fp32 geometry (8 heads of 64, no grouping) at its prompt length
        dict(name="packed f32", op="packed", dtype=F32, hq=8, hkv=8, d=64, n_seq=5, max_len=2048,
             layout="heads", lens=4),
        # the chat batch's keys and values enter the cache
        dict(name="load chat bf16", op="load", dtype=BF16, hq=32, hkv=8, d=128, n_seq=24, max_len=1024,
             layout="tokens", lens=2, window=256, block=32),
        # long documents enter the cache of a larger batch
        dict(name="load long bf16", op="load", dtype=BF16, hq=32, hkv=8, d=128, n_seq=8, max_len=32768,
             layout="heads", lens=5, window=4096, block=128),
        # four drafted tokens over a short conversation: latency
        dict(name="tree short bf16", op="tree", dtype=BF16, hq=32, hkv=8, d=128, batch=1, T=4, ctx=600,
             keep=1.0, window=256, block=32, shape="chain", lens=6),
        # sixteen drafted tokens for each of four sequences over compressed 32K prompts
        dict(name="tree 32K x4 bf16", op="tree", dtype=BF16, hq=32, hkv=8, d=128, batch=4, T=16, ctx=32768,
             keep=0.32, window=4096, block=128, shape="bushy", lens=7),
        # a wide tree over one compressed 128K prompt
        dict(name="tree 128K bf16", op="tree", dtype=BF16, hq=32, hkv=8, d=128, batch=1, T=64, ctx=131072,
             keep=0.32, window=4096, block=128, shape="bushy", lens=8),
        # the fp32 geometry
        dict(name="tree f32", op="tree", dtype=F32, hq=8, hkv=8, d=64, batch=2, T=13, ctx=2048, keep=0.5,
             window=128, block=32, shape="bushy", lens=9),
        # a few tokens accepted by each of four sequences, one or two of which compress a block
        dict(name="accept x4 bf16", op="accept", dtype=BF16, hq=32, hkv=8, d=128, batch=4, T=16, window=4096,
             block=128, near=0.3, lens=10),
        # a busy server: 64 sequences accept up to 32 tokens, most of them compress
        dict(name="accept x64 bf16", op="accept", dtype=BF16, hq=32, hkv=8, d=128, batch=64, T=32, window=1024,
             block=128, near=0.9, lens=11),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["packed", "packed", "load", "tree", "tree", "accept"])
    dtype = BF16 if rng.random() < 0.75 else F32
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.randint(1, 32 // hkv if hkv > 4 else 8)
    d = rng.choice([64, 128])
    c = dict(op=op, dtype=dtype, hq=hq, hkv=hkv, d=d, lens=rng.randrange(1 << 20))
    if op in ("packed", "load"):
        top = 8192 if dtype == BF16 else 2048
        if op == "load":
            top = 32768
        c.update(n_seq=_log(rng, 1, 32), max_len=_log(rng, 1, top), layout=rng.choice(["heads", "tokens"]))
        if op == "packed":      # no more than the largest listed case's padded square
            c["n_seq"] = max(1, min(c["n_seq"], 3 * 8192 * 8192 // (c["max_len"] * c["max_len"])))
        else:
            c["n_seq"] = max(1, min(c["n_seq"], 8 * 32768 // c["max_len"]))
            c.update(block=rng.choice([16, 32, 64, 128]), window=_log(rng, 1, 4096))
    elif op == "tree":
        batch = _log(rng, 1, 8)
        ctx = _log(rng, 1, 131072 // batch if dtype == BF16 else 8192 // batch)
        c.update(batch=batch, T=_log(rng, 1, 64), ctx=ctx, keep=round(rng.uniform(0.05, 0.32), 3),
                 block=rng.choice([16, 32, 64, 128]), window=_log(rng, 1, 4096), shape=rng.choice(["chain", "bushy"]))
    else:
        block = rng.choice([32, 64, 128])
        c.update(batch=_log(rng, 1, 64), T=_log(rng, 1, 32), block=block, window=_log(rng, 128, 1024),
                 near=round(rng.random(), 2))
    return c


# ------------------------------------------------------------------ sizes that follow from a case alone
def _lengths(c):
    """Prompt lengths: the longest first drawn, the others log-uniform below it, one of four or more empty."""
    r = random.Random(c["lens"])
    lens = [c["max_len"]] + [_log(r, 1, c["max_len"]) for _ in range(c["n_seq"] - 1)]
    if len(lens) >= 4:
        lens[2] = 0
    r.shuffle(lens)
    return lens


def _starts(lens):
    s = np.zeros(len(lens) + 1, dtype=np.int64)
    s[1:] = np.cumsum(lens)
    return s


def _packed_rows(c):
    """Rows of the packed buffers: five more than the sequences have (padding a batch is common)."""
    return sum(_lengths(c)) + 5


def _load_cache(c):
    """Cache of a load case: one more sequence than prompts; capacities of the longest prompt, slots shuffled."""
    lens, w, b = _lengths(c), c["window"], c["block"]
    r = random.Random(c["lens"] + 1)
    slots = list(range(c["n_seq"] + 1))
    r.shuffle(slots)
    slots = slots[:c["n_seq"]]
    cap = [0] * (c["n_seq"] + 1)
    for s, n in zip(slots, lens):
        cap[s] = max(0, (n - w) // b) * b
    return np.array(slots, dtype=np.int32), np.repeat(np.array(cap, dtype=np.int64), c["hkv"])


def _segments(gcap, tail_cap):
    seg = np.zeros(len(gcap), dtype=np.int64)
    seg[1:] = np.cumsum(gcap[:-1] + tail_cap)
    return seg, int(seg[-1] + gcap[-1] + tail_cap)


def _retained(c):
    """Host mirror of the retained cache of a tree or accept case, per unit (sequence, KV head)."""
    r = random.Random(c["lens"])
    B, H, w, b = c["batch"], c["hkv"], c["window"], c["block"]
    tail_cap = w + b + TREE_MAX
    U = B * H
    keep = np.zeros(U, dtype=np.int64)
    n_glob, head, tail, seq = (np.zeros(U, dtype=np.int64) for _ in range(4))
    for s in range(B):
        if c["op"] == "tree":
            L = max(1, c["ctx"] - (r.randrange(max(1, c["ctx"] // 8)) if s else 0))
            m = max(0, (L - w) // b)
            n_tail = L - m * b
        else:
            m = 4
            n_tail = w + b - (r.randint(1, min(c["T"], b)) if r.random() < c["near"] else r.randint(c["T"] + 1, w))
            L = m * b + n_tail
        hd = r.randrange(tail_cap)
        for h in range(H):
            u = s * H + h
            frac = min(1.0, c.get("keep", 0.3) * r.uniform(0.4, 1.6)) if c.get("keep", 0.3) < 1.0 else 1.0
            keep[u] = min(b, max(1, int(frac * b)))
            n_glob[u] = min(m * b, int(frac * m * b))
            head[u], tail[u], seq[u] = hd, n_tail, L
    gcap = n_glob + 2 * keep
    seg, rows = _segments(gcap, tail_cap)
    return dict(U=U, tail_cap=tail_cap, keep=keep, n_global=n_glob, tail_head=head, n_tail=tail, seq_len=seq,
                gcap=gcap, seg=seg, rows=rows)


def _drafts(c):
    """Parents [batch, T] and drafted counts [batch] of a tree case (some sequences drafted fewer)."""
    r = random.Random(c["lens"] + 2)
    T = c["T"]
    par = np.full((c["batch"], T), -1, dtype=np.int32)
    n = np.full(c["batch"], T, dtype=np.int32)
    for s in range(c["batch"]):
        for t in range(T):
            if c["shape"] == "chain":
                par[s, t] = t - 1
            else:
                par[s, t] = r.randint(max(-1, (t - 4) // 3 - 1), max(-1, t // 2 - 1)) if t > 3 else -1
        if s % 2:
            n[s] = max(1, T - r.randrange(T))
    return par, n


def _accepted(c):
    """Paths [batch, T] and accepted counts [batch]: ascending drafted indices, 1 .. min(T, block) of them."""
    r = random.Random(c["lens"] + 3)
    T = c["T"]
    path = np.zeros((c["batch"], T), dtype=np.int32)
    n = np.zeros(c["batch"], dtype=np.int32)
    for s in range(c["batch"]):
        n[s] = r.randint(1, min(T, c["block"])) if s % 5 != 4 else 0
        path[s, :n[s]] = sorted(r.sample(range(T), int(n[s])))
    return path, n


def _scale(c):
    return float(np.float32(1.0 / math.sqrt(c["d"])))


def _dt(c):
    return torch.bfloat16 if c["dtype"] == BF16 else torch.float32


# ------------------------------------------------------------------ inputs
def _randn(gen, shape, c, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std).to(_dt(c))


def _packed_tensor(gen, heads, rows, c):
    """[heads, rows, d], head-major, or a view of a token-major [rows, heads, d] buffer."""
    if c["layout"] == "heads":
        return _randn(gen, (heads, rows, c["d"]), c)
    return _randn(gen, (rows, heads, c["d"]), c).transpose(0, 1)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(c=c, scale=_scale(c))
    G = c["hq"] // c["hkv"]
    if c["op"] in ("packed", "load"):
        rows = _packed_rows(c)
        s["start_host"] = _starts(_lengths(c))
        s["start"] = torch.from_numpy(s["start_host"]).cuda()
        s["k"] = _packed_tensor(gen, c["hkv"], rows, c)
        s["v"] = _packed_tensor(gen, c["hkv"], rows, c)
        if c["op"] == "packed":
            s["q"] = _packed_tensor(gen, c["hq"], rows, c)
            s["o"] = torch.zeros_like(s["q"])
        else:
            s["slots"], gcap = _load_cache(c)
            tail_cap = c["window"] + c["block"]
            seg, rows_c = _segments(gcap, tail_cap)
            U = len(gcap)
            zero = np.zeros(U, dtype=np.int64)
            s["mirror"] = dict(U=U, tail_cap=tail_cap, keep=zero, n_global=zero, tail_head=zero, n_tail=zero,
                               seq_len=zero, gcap=gcap, seg=seg, rows=rows_c)
            s["cache"] = _cache_tensors(s["mirror"], c, None)
    else:
        s["mirror"] = _retained(c)
        s["cache"] = _cache_tensors(s["mirror"], c, gen)
        B, T = c["batch"], c["T"]
        s["q"] = _randn(gen, (B, c["hq"], T, c["d"]), c, 1.5)
        s["kd"] = _randn(gen, (B, c["hkv"], T, c["d"]), c)
        s["vd"] = _randn(gen, (B, c["hkv"], T, c["d"]), c)
        if c["op"] == "tree":
            par, n = _drafts(c)
            s["parent"], s["n_draft"] = torch.from_numpy(par).cuda(), torch.from_numpy(n).cuda()
            s["o"] = torch.zeros_like(s["q"])
        else:
            s["path_host"], s["n_accept"] = _accepted(c)
            s["path"] = torch.from_numpy(s["path_host"]).cuda()
            s["state0"] = s["cache"]["state"].clone()
    if own:
        _handles(s)
    return s


def _cache_tensors(m, c, gen):
    """The cache's buffers: rows [rows, d], positions, and the state words of every unit."""
    dev = "cuda"
    if gen is None:
        k = torch.zeros(m["rows"], c["d"], dtype=_dt(c), device=dev)
        v = torch.zeros_like(k)
    else:
        k, v = _randn(gen, (m["rows"], c["d"]), c), _randn(gen, (m["rows"], c["d"]), c)
    pos = torch.full((m["rows"],), -1, dtype=torch.int32, device=dev)
    st = np.zeros((m["U"], STATE_WORDS), dtype=np.int64)
    for i, key in enumerate(("seg", "gcap", "n_global", "tail_head", "n_tail", "seq_len", "keep")):
        st[:, i] = m[key]
    if gen is not None:   # positions: the global rows ascending from 0, the ring the last n_tail tokens
        r = torch.arange(m["rows"], device=dev)
        u = torch.bucketize(r, torch.from_numpy(m["seg"]).to(dev), right=True) - 1
        t = {x: torch.from_numpy(m[x]).to(dev)[u] for x in ("seg", "gcap", "n_global", "tail_head", "n_tail", "seq_len")}
        local = r - t["seg"]
        ring = torch.remainder(local - t["gcap"] - t["tail_head"], m["tail_cap"])
        pos = torch.where(local < t["n_global"], local, pos)
        pos = torch.where((local >= t["gcap"]) & (ring < t["n_tail"]), t["seq_len"] - t["n_tail"] + ring, pos).int()
    return dict(k=k, v=v, pos=pos, state=torch.from_numpy(st.reshape(-1)).to(dev))


def _handles(s):
    """What a program that uses the library keeps: parameters, workspace, cache handle."""
    from paper_2512_09238_b200 import binding as B
    c = s["c"]
    dt = B.TCA_BF16 if c["dtype"] == BF16 else B.TCA_F32
    batch = c.get("batch", c.get("n_seq"))
    if c["op"] == "load":
        batch = c["n_seq"] + 1
    s["prm"] = B.make_params(batch, c["hq"], c["hkv"], c["d"], c.get("block", 128), c.get("window", 128),
                             sm_scale=s["scale"], dtype=dt)
    if "mirror" in s:
        m, t = s["mirror"], s["cache"]
        h = B.Cache(s["prm"], m["gcap"], m["tail_cap"], m["keep"], init=False)
        for name in ("n_global", "tail_head", "n_tail", "seq_len"):
            getattr(h, name)[:] = m[name]
        B.tca_cache_init(s["prm"], h)
        h.k.copy_(t["k"])
        h.v.copy_(t["v"])
        h.pos.copy_(t["pos"])
        s["handle"] = h
        s["cache"] = dict(k=h.k, v=h.v, pos=h.pos, state=h.state)
    if c["op"] == "packed":
        s["ws"] = B.alloc_workspace(s["prm"], s["q"].shape[1], B.TCA_OP_PACKED)
    elif c["op"] == "tree":
        s["ws"] = B.alloc_tree_workspace(s["prm"], c["T"])


# ------------------------------------------------------------------ one pass
def run(state):
    s = state
    op = s["c"]["op"]
    if own:
        from paper_2512_09238_b200 import binding as B
        if op == "packed":
            B.tca_attn_packed(s["prm"], s["q"], s["k"], s["v"], s["q"].shape[1], s["start"], s["o"], s["ws"])
            return s["o"]
        if op == "load":
            B.tca_cache_load(s["prm"], s["k"], s["v"], s["k"].shape[1], s["start_host"], s["slots"], s["handle"])
            return dict(s["cache"])
        if op == "tree":
            B.tca_attn_tree(s["prm"], s["q"], s["kd"], s["vd"], s["c"]["T"], s["parent"], s["n_draft"], s["handle"],
                            s["o"], s["ws"])
            return s["o"]
        # every pass accepts from the same cache: lengths go back to where the draft was made
        s["cache"]["state"].copy_(s["state0"])
        for name in ("n_global", "tail_head", "n_tail", "seq_len"):
            getattr(s["handle"], name)[:] = s["mirror"][name]
        B.tca_cache_accept(s["prm"], s["handle"], s["kd"], s["vd"], s["q"], s["c"]["T"], s["path"], s["n_accept"])
        return dict(s["cache"])
    if op == "packed":
        return _plain_packed(s)
    if op == "load":
        return _plain_load(s)
    if op == "tree":
        return _plain_tree(s)
    s["cache"]["state"].copy_(s["state0"])
    return _plain_accept(s)


def _plain_packed(s):
    """Sequences padded to the longest; all heads and sequences in one product."""
    c, o = s["c"], s["o"]
    n, Lm, G, d = c["n_seq"], c["max_len"], c["hq"] // c["hkv"], c["d"]
    start = s["start"]
    i = torch.arange(Lm, device="cuda")
    inside = i[None, :] < (start[1:] - start[:-1])[:, None]                      # [n, Lm]
    row = torch.where(inside, start[:-1, None] + i, 0)
    q = s["q"][:, row].float().view(c["hkv"], G, n, Lm, d).permute(2, 0, 1, 3, 4).reshape(n, c["hkv"], G * Lm, d)
    k = s["k"][:, row].float().permute(1, 0, 2, 3)                               # [n, hkv, Lm, d]
    v = s["v"][:, row].float().permute(1, 0, 2, 3)
    x = (q * s["scale"]) @ k.transpose(-1, -2)
    x = x.view(n, c["hkv"], G, Lm, Lm)
    x.masked_fill_(i[None, :] > i[:, None], float("-inf"))
    x.sub_(x.amax(-1, keepdim=True)).exp_()
    total = x.sum(-1, keepdim=True)
    out = (x.view(n, c["hkv"], G * Lm, Lm) @ v).view(n, c["hkv"], G, Lm, d) / total
    out = out.permute(1, 2, 0, 3, 4).reshape(c["hq"], n, Lm, d).to(o.dtype)
    # rows of no sequence keep what they held
    r = torch.arange(o.shape[1], device="cuda")
    seq = torch.clamp(torch.bucketize(r, start, right=True) - 1, 0, n - 1)
    of_seq = (r >= start[0]) & (r < start[-1])
    o.copy_(torch.where(of_seq[None, :, None], out[:, seq, torch.where(of_seq, r - start[seq], 0)], o))
    return o


def _plain_load(s):
    c, m, t = s["c"], s["mirror"], s["cache"]
    H, w, b = c["hkv"], c["window"], c["block"]
    start = s["start_host"]
    lens = start[1:] - start[:-1]
    nb = np.maximum(0, (lens - w) // b) * b
    seq = np.repeat(np.arange(c["n_seq"]), lens)
    p = np.arange(start[-1]) - start[seq]
    unit = s["slots"][seq].astype(np.int64)[None, :] * H + np.arange(H)[:, None]   # [H, tokens]
    dst = m["seg"][unit] + np.where(p < nb[seq], p, m["gcap"][unit] + p - nb[seq])
    dst = torch.from_numpy(dst).cuda()
    n = int(start[-1])
    t["k"][dst] = s["k"][:, :n]
    t["v"][dst] = s["v"][:, :n]
    t["pos"][dst] = torch.from_numpy(np.broadcast_to(p, dst.shape).astype(np.int32)).cuda()
    words = torch.from_numpy(np.stack([nb, np.zeros_like(nb), lens - nb, lens], 1)).cuda()   # n_global .. seq_len
    units = torch.from_numpy(s["slots"].astype(np.int64)[:, None] * H + np.arange(H)).cuda()
    t["state"].view(-1, STATE_WORDS)[:, 2:6][units] = words[:, None, :]
    return dict(t)


def _rows_of(state, tail_cap, n):
    """Physical rows [U, n] of every unit in logical order and which of them exist."""
    seg, gcap, ng, head, nt = (state.view(-1, STATE_WORDS)[:, i, None] for i in range(5))
    r = torch.arange(n, device="cuda")[None, :]
    ring = torch.remainder(head + r - ng, tail_cap)
    there = r < ng + nt
    return torch.where(there, torch.where(r < ng, seg + r, seg + gcap + ring), seg), there


def _plain_tree(s):
    c, m, t = s["c"], s["mirror"], s["cache"]
    B, H, G, T, d = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["T"], c["d"]
    rows, there = _rows_of(t["state"], m["tail_cap"], int((m["n_global"] + m["n_tail"]).max()))
    k, v = t["k"][rows].float(), t["v"][rows].float()                              # [U, N, d]
    v = v.masked_fill(~there[:, :, None], 0.0)
    q = s["q"].float().reshape(B * H, G * T, d) * s["scale"]
    kd, vd = s["kd"].float().reshape(B * H, T, d), s["vd"].float().reshape(B * H, T, d)
    up = (s["parent"][:, :, None] == torch.arange(T, device="cuda")).double()     # up[t, parent of t] = 1
    eye = torch.eye(T, device="cuda", dtype=torch.float64)
    sees = torch.linalg.matrix_power(up + eye, T) > 0                              # [B, T, T] path to the root
    sees = sees[:, None, None].expand(B, H, G, T, T).reshape(B * H, G * T, T)
    x = (q @ k.transpose(-1, -2)).masked_fill(~there[:, None, :], float("-inf"))
    y = (q @ kd.transpose(-1, -2)).masked_fill(~sees, float("-inf"))
    top = torch.maximum(x.amax(-1, keepdim=True), y.amax(-1, keepdim=True))
    x, y = (x - top).exp(), (y - top).exp()
    out = (x @ v + y @ vd) / (x.sum(-1, keepdim=True) + y.sum(-1, keepdim=True))
    out = out.view(B, c["hq"], T, d).to(s["o"].dtype)
    live = torch.arange(T, device="cuda")[None, :] < s["n_draft"][:, None]
    s["o"].copy_(torch.where(live[:, None, :, None], out, s["o"]))
    return s["o"]


def _plain_accept(s):
    """At most one block leaves a ring in a pass: no more than `block` tokens are accepted."""
    c, m, t = s["c"], s["mirror"], s["cache"]
    B, H, G, T, d, w, b = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["T"], c["d"], c["window"], c["block"]
    U, cap = m["U"], m["tail_cap"]
    n = np.repeat(s["n_accept"].astype(np.int64), H)                               # per unit
    ring = m["seg"] + m["gcap"]
    # the accepted rows
    u = np.repeat(np.arange(U), n)
    i = np.arange(len(u)) - np.repeat(np.cumsum(n) - n, n)
    src = u * T + s["path_host"][u // H, i]
    dst = ring[u] + (m["tail_head"][u] + m["n_tail"][u] + i) % cap
    if len(u):
        src_t, dst_t = torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda()
        t["k"][dst_t] = s["kd"].reshape(U * T, d)[src_t]
        t["v"][dst_t] = s["vd"].reshape(U * T, d)[src_t]
        t["pos"][dst_t] = torch.from_numpy((m["seq_len"][u] + i).astype(np.int32)).cuda()
    # the units whose ring reached window + block, and the token that made it so
    full = np.nonzero(m["n_tail"] + n >= w + b)[0]
    state = np.stack([m[x] for x in ("seg", "gcap", "n_global", "tail_head", "n_tail", "seq_len", "keep")]
                     + [np.zeros(U, dtype=np.int64)], 1)
    state[:, 4] += n
    state[:, 5] += n
    if len(full):
        at = w + b - 1 - m["n_tail"][full]
        tok = s["path_host"][full // H, at]
        blk = ring[full][:, None] + (m["tail_head"][full][:, None] + np.arange(b)) % cap
        blk = torch.from_numpy(blk).cuda()
        f = torch.from_numpy(full).cuda()
        q = s["q"].view(U, G, T, d)[f, :, torch.from_numpy(tok).cuda().long()].double()   # [F, G, d]
        x = (q @ t["k"][blk].double().transpose(-1, -2)) * s["scale"]              # [F, G, b]
        x = x - torch.logsumexp(x, -1, keepdim=True)
        score = torch.logsumexp(x, 1) if G > 1 else x[:, 0]
        order = torch.sort(score, dim=-1, descending=True, stable=True)[1]         # ties to the older token
        keep = m["keep"][full]
        rank = torch.empty_like(order).scatter_(1, order, torch.arange(b, device="cuda").expand_as(order).contiguous())
        kept = rank < torch.from_numpy(keep).cuda()[:, None]
        place = torch.sort((~kept).to(torch.int8), dim=-1, stable=True)[1]         # the kept ones first, in order
        a = np.repeat(np.arange(len(full)), keep)
        r = np.arange(len(a)) - np.repeat(np.cumsum(keep) - keep, keep)
        a_t = torch.from_numpy(a).cuda()
        src = blk[a_t, place[a_t, torch.from_numpy(r).cuda()]]
        dst = torch.from_numpy(m["seg"][full][a] + m["n_global"][full][a] + r).cuda()
        for name in ("k", "v", "pos"):
            t[name][dst] = t[name][src]
        state[full, 2] += keep
        state[full, 3] = (state[full, 3] + b) % cap
        state[full, 4] -= b
    t["state"].copy_(torch.from_numpy(state.reshape(-1)))
    return dict(t)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    e = 2 if c["dtype"] == BF16 else 4
    G = c["hq"] // c["hkv"]
    if c["op"] == "packed":
        lens = _lengths(c)
        rows = sum(lens)
        pairs = sum(n * (n + 1) // 2 for n in lens)
        return dict(bytes=rows * c["d"] * e * (2 * c["hq"] + 2 * c["hkv"]), flops=4 * c["d"] * c["hq"] * pairs)
    if c["op"] == "load":
        rows = sum(_lengths(c)) * c["hkv"]
        return dict(bytes=2 * 2 * rows * c["d"] * e + 4 * rows, flops=0)
    m = _retained(c)
    if c["op"] == "tree":
        par, n = _drafts(c)
        rows = int((m["n_global"] + m["n_tail"]).sum())
        live = int(n.sum())
        depth = 0
        for s in range(c["batch"]):
            deep = []
            for t in range(int(n[s])):
                deep.append(1 + (deep[par[s, t]] if par[s, t] >= 0 else 0))
            depth += sum(deep)
        per = np.repeat(n, c["hkv"]).astype(np.int64)
        keys = int(((m["n_global"] + m["n_tail"]) * per).sum()) * G + depth * c["hq"]
        return dict(bytes=c["d"] * e * (2 * rows + 2 * live * c["hq"] + 2 * live * c["hkv"]), flops=4 * c["d"] * keys)
    path, n = _accepted(c)
    per = np.repeat(n, c["hkv"]).astype(np.int64)
    full = m["n_tail"] + per >= c["window"] + c["block"]
    moved = int(m["keep"][full].sum())
    rows = 4 * int(per.sum()) + int(full.sum()) * (c["block"] + G) + 3 * moved
    return dict(bytes=rows * c["d"] * e + 2 * 64 * m["U"], flops=2 * c["d"] * G * c["block"] * int(full.sum()))


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    c = dict(case)
    global own
    keep_own, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = keep_own
    G, d, scale = c["hq"] // c["hkv"], c["d"], s["scale"]
    if c["op"] == "packed":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lens = _lengths(c)
        for i, n in enumerate(lens):
            lo = int(sum(lens[:i]))
            tri = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
            for h in range(c["hq"] if n else 0):
                q, k, v = (x[y, lo:lo + n].double() for x, y in ((s["q"], h), (s["k"], h // G), (s["v"], h // G)))
                p = torch.softmax((q @ k.T * scale).where(tri, torch.tensor(-math.inf, dtype=torch.float64, device="cuda")), -1)
                out[h, lo:lo + n] = p @ v
        return out
    t, m = s["cache"], s["mirror"]
    H = c["hkv"]
    if c["op"] == "load":
        k, v = t["k"].double(), t["v"].double()
        lo = 0
        for i, n in enumerate(_lengths(c)):
            g = max(0, (n - c["window"]) // c["block"]) * c["block"]
            for h in range(H):
                u = int(s["slots"][i]) * H + h
                a = int(m["seg"][u])
                z = a + int(m["gcap"][u])
                for to, x in ((k, s["k"]), (v, s["v"])):
                    to[a:a + g] = x[h, lo:lo + g].double()
                    to[z:z + n - g] = x[h, lo + g:lo + n].double()
            lo += n
        return dict(k=k, v=v, pos=None, state=None)
    cap, T = m["tail_cap"], c["T"]

    def ring_rows(u, first, n):
        at = (int(m["tail_head"][u]) + first + torch.arange(n, device="cuda")) % cap
        return int(m["seg"][u] + m["gcap"][u]) + at

    if c["op"] == "tree":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        par, nd = _drafts(c)
        for b in range(c["batch"]):
            line = torch.zeros(T, T, dtype=torch.bool)
            for i in range(T):
                j = i
                while j >= 0:
                    line[i, j] = True
                    j = int(par[b, j])
            line = line.cuda()
            n = int(nd[b])
            for h in range(H):
                u = b * H + h
                rows = torch.cat([int(m["seg"][u]) + torch.arange(int(m["n_global"][u]), device="cuda"),
                                  ring_rows(u, 0, int(m["n_tail"][u]))])
                k = torch.cat([t["k"][rows], s["kd"][b, h]]).double()
                v = torch.cat([t["v"][rows], s["vd"][b, h]]).double()
                vis = torch.cat([torch.ones(T, len(rows), dtype=torch.bool, device="cuda"), line], 1)
                for g in range(G):
                    x = s["q"][b, h * G + g].double() @ k.T * scale
                    p = torch.softmax(x.masked_fill(~vis, -math.inf), -1)
                    out[b, h * G + g, :n] = (p @ v)[:n]
        return out
    k, v = t["k"].double(), t["v"].double()
    path, na = _accepted(c)
    for u in range(m["U"]):
        b = u // H
        n_tail, w, blk = int(m["n_tail"][u]), c["window"], c["block"]
        n = int(na[b])
        if n == 0:
            continue
        tok = torch.from_numpy(path[b, :n]).cuda().long()
        dst = ring_rows(u, n_tail, n)
        k[dst], v[dst] = s["kd"][b, u % H][tok].double(), s["vd"][b, u % H][tok].double()
        if n_tail + n >= w + blk:
            old = ring_rows(u, 0, blk)
            q = s["q"][b, (u % H) * G:(u % H + 1) * G, int(path[b, w + blk - 1 - n_tail])].double()
            p = torch.softmax(q @ k[old].T * scale, -1).mean(0)
            best = torch.topk(p, int(m["keep"][u]))[1].sort()[0]
            to = int(m["seg"][u] + m["n_global"][u])
            k[to:to + len(best)], v[to:to + len(best)] = k[old[best]], v[old[best]]
    return dict(k=k, v=v, pos=None, state=None)
