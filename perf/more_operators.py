"""Workloads of the paged-cache operators: prompt attention with a sliding window and sink tokens, appending to a
paged cache, attention of one new token over it, and eviction by accumulated attention weight.

``listed()`` and ``draw()`` name cases, ``prepare()`` makes their inputs, ``run()`` is one call of the operator: in
its plain form (elementary torch operations, 32 bits or more, rounded once at the end) or, where ``own`` is set,
through the library.  ``exact()`` is the operator's definition in 64 bits.  ``work()`` states the bytes and
floating-point operations a pass cannot do without.

Definitions (0-based; scale = 1/sqrt(head_dim) as a float32; a unit is one (sequence, KV head) pair; the rows of a
unit lie in slots 0 .. len-1, slot j in row j % page_size of page table[unit][j // page_size]):
  window  sequence s owns rows [start[s], start[s+1]); row i of it attends to its rows j <= i with i - j < window or
          j < n_sink.
  append  row i of a sequence's new rows goes to slot len + i of each of its units, with position next + i and the
          given attention weight (or 0); len and next grow by the number of rows.
  paged   a unit's query heads attend to the slots j < len with j >= len - window or j < n_sink; where weights are
          accumulated, a visible row's mass grows by the mean over the unit's query heads of its softmax weight.
  evict   a unit with more than budget rows keeps budget of them: the slots below n_sink, the rows whose position is
          above the unit's largest minus n_recent, and those of the others with the largest mass (ties to the lower
          slot).  Kept rows in slots below budget stay; the other kept rows fill the evicted slots below budget, both
          in ascending order of slots.
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F32 = "bf16", "f32"
ALL = (1 << 31) - 1     # a window that hides nothing


# ------------------------------------------------------------------ cases
def listed():
    return [
        # three short prompts that arrive together at a layer with a small window: latency
        dict(name="window short bf16", op="window", dtype=BF16, hq=32, hkv=8, d=128, n_seq=3, max_len=300, window=128,
             n_sink=4, layout="heads", lens=1),
        # a batch of chat turns of very different lengths, token-major as a fused projection writes it
        dict(name="window chat bf16", op="window", dtype=BF16, hq=32, hkv=8, d=128, n_seq=24, max_len=2048, window=512,
             n_sink=16, layout="tokens", lens=2),
        # long documents under the window of the retained-cache layers
        dict(name="window long bf16", op="window", dtype=BF16, hq=32, hkv=8, d=128, n_seq=3, max_len=32768, window=4096,
             n_sink=4, layout="heads", lens=3),
        # the fp32 geometry (8 heads of 64, no grouping)
        dict(name="window f32", op="window", dtype=F32, hq=8, hkv=8, d=64, n_seq=5, max_len=2048, window=300, n_sink=8,
             layout="heads", lens=4),
        # the tokens of one decode step of 64 sequences
        dict(name="append step bf16", op="append", dtype=BF16, hq=32, hkv=8, d=128, batch=64, ctx=1500, new=1, page=32,
             layout="heads", lens=5),
        # prompts of up to 8K tokens join a batch, with the weights that their prefill gave them
        dict(name="append prompts bf16", op="append", dtype=BF16, hq=32, hkv=8, d=128, batch=16, ctx=100, new=8192,
             page=64, layout="tokens", lens=6),
        # one short conversation: latency
        dict(name="paged short bf16", op="paged", dtype=BF16, hq=32, hkv=8, d=128, batch=1, ctx=700, page=16, window=ALL,
             n_sink=0, mass=False, lens=7),
        # a busy server: 64 conversations of up to 4K tokens, weights accumulated for a later eviction
        dict(name="paged x64 mass bf16", op="paged", dtype=BF16, hq=32, hkv=8, d=128, batch=64, ctx=4096, page=32,
             window=ALL, n_sink=0, mass=True, lens=8),
        # four long documents
        dict(name="paged long bf16", op="paged", dtype=BF16, hq=32, hkv=8, d=128, batch=4, ctx=65536, page=128, window=ALL,
             n_sink=0, mass=False, lens=9),
        # the fp32 geometry under a window, weights accumulated
        dict(name="paged window f32", op="paged", dtype=F32, hq=8, hkv=8, d=64, batch=8, ctx=8192, page=64, window=1000,
             n_sink=4, mass=True, lens=10),
        # a few conversations a little over their budgets
        dict(name="evict x4 bf16", op="evict", dtype=BF16, hq=32, hkv=8, d=128, batch=4, ctx=1200, page=16, n_sink=4,
             n_recent=128, keep=0.9, lens=11),
        # long documents cut to a third
        dict(name="evict long bf16", op="evict", dtype=BF16, hq=32, hkv=8, d=128, batch=4, ctx=65536, page=64, n_sink=4,
             n_recent=1024, keep=0.33, lens=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "window", "append", "paged", "paged", "paged", "evict"])
    dtype = BF16 if rng.random() < 0.75 else F32
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.randint(1, 32 // hkv if hkv > 4 else 8)
    c = dict(op=op, dtype=dtype, hq=hq, hkv=hkv, d=rng.choice([64, 128]), lens=rng.randrange(1 << 20))
    if op == "window":
        max_len = _log(rng, 1, 32768 if dtype == BF16 else 4096)
        window = _log(rng, 1, 4096)
        most = 3 * 32768 * 4096 // (32 if dtype == F32 else 1)
        n = max(1, min(_log(rng, 1, 32), most // (max_len * min(window, max_len))))
        c.update(n_seq=n, max_len=max_len, window=window, n_sink=rng.choice([0, 1, 4, rng.randint(1, 300)]),
                 layout=rng.choice(["heads", "tokens"]))
        return c
    batch = _log(rng, 1, 64)
    c.update(batch=batch, page=rng.choice([16, 32, 64, 128, 256]))
    if op == "append":
        c.update(ctx=_log(rng, 1, 2048), new=rng.choice([1, _log(rng, 1, 65536 // batch)]),
                 layout=rng.choice(["heads", "tokens"]))
    elif op == "paged":
        c.update(ctx=_log(rng, 1, 262144 // batch // (1 if dtype == BF16 else 4)), mass=rng.random() < 0.5,
                 window=rng.choice([ALL, _log(rng, 1, 4096)]), n_sink=rng.choice([0, 1, 4, rng.randint(1, 300)]))
    else:
        ctx = _log(rng, 8, 262144 // batch // (1 if dtype == BF16 else 4))
        c.update(ctx=ctx, n_sink=rng.choice([0, 1, 4]), n_recent=rng.randint(0, max(0, ctx // 8)),
                 keep=round(rng.uniform(0.3, 0.95), 3))
    return c


# ------------------------------------------------------------------ sizes that follow from a case alone
def _lengths(c, n, longest):
    """The longest first drawn, the others log-uniform below it, one of four or more empty."""
    r = random.Random(c["lens"])
    lens = [longest] + [_log(r, 1, longest) for _ in range(n - 1)]
    if len(lens) >= 4 and longest > 1:
        lens[2] = 0
    r.shuffle(lens)
    return lens


def _starts(lens):
    s = np.zeros(len(lens) + 1, dtype=np.int64)
    s[1:] = np.cumsum(lens)
    return s


def _window_lens(c):
    return _lengths(c, c["n_seq"], c["max_len"])


def _unit_lens(c):
    """Rows of every unit [batch * hkv]: those of a sequence differ a little between heads, as per-head budgets leave them."""
    r = random.Random(c["lens"] + 1)
    out = []
    for n in _lengths(c, c["batch"], c["ctx"]):
        out += [n if c["op"] == "append" or n == 0 else max(1, n - r.randrange(1 + n // 8)) for _ in range(c["hkv"])]
    return np.array(out, dtype=np.int64)


def _new_lens(c):
    """New rows of every sequence of an append case."""
    if c["new"] == 1:
        return [1] * c["batch"]
    return _lengths(dict(lens=c["lens"] + 2), c["batch"], c["new"])


def _budgets(c):
    r = random.Random(c["lens"] + 3)
    lens = _unit_lens(c)
    return np.array([max(c["n_sink"] + c["n_recent"], int(n * min(1.0, c["keep"] * r.uniform(0.8, 1.2)))) for n in lens],
                    dtype=np.int32)


def _visible(c, n):
    """Slots of a unit of n rows that the new token sees: [0, sinks) and [lo, n)."""
    lo = np.maximum(0, n - c["window"])
    return np.minimum(c["n_sink"], lo), lo


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


def _pool(c, gen, seed, lens, room):
    """A paged cache whose units hold `lens` rows in pages dealt at random, with room for `room` rows each."""
    ps, U = c["page"], len(lens)
    need = -(-np.maximum(room, 1) // ps)
    n_pages, max_pages = int(need.sum()) + 3, int(need.max()) + 1
    rng = np.random.default_rng(seed)
    order = rng.permutation(n_pages)
    table = np.full((U, max_pages), -1, dtype=np.int32)
    at = 0
    for u in range(U):
        table[u, :need[u]] = order[at:at + need[u]]
        at += need[u]
    k, v = _randn(gen, (n_pages, ps, c["d"]), c), _randn(gen, (n_pages, ps, c["d"]), c)
    # one buffer of 32-bit words: positions, masses, then four state words a unit (rows, next position, 0, 0)
    meta = torch.zeros(2 * n_pages * ps + 4 * U, dtype=torch.int32, device="cuda")
    p = dict(k=k, v=v, meta=meta, pos=meta[:n_pages * ps].view(n_pages, ps),
             mass=meta[n_pages * ps:2 * n_pages * ps].view(torch.float32).view(n_pages, ps),
             state=meta[2 * n_pages * ps:].view(U, 4), table=torch.from_numpy(table).cuda())
    # weights: heavy-tailed, some exactly zero; positions: those of a cache that has dropped a quarter of what it saw
    mass = torch.randn(n_pages, ps, generator=gen, device="cuda").mul_(2.0).exp_()
    mass.masked_fill_(torch.rand(n_pages, ps, generator=gen, device="cuda") < 0.05, 0.0)
    p["mass"].copy_(mass)
    st = np.zeros((U, 4), dtype=np.int32)
    slot_pos = np.full((U, int(lens.max()) if U else 0), -1, dtype=np.int32)
    keep_first = c.get("n_sink", 0)
    for u in range(U):
        n = int(lens[u])
        seen = n + n // 3 if c["op"] == "evict" else n
        st[u, 0], st[u, 1] = n, seen
        x = np.arange(n)
        if seen > n:
            x[keep_first:] = keep_first + np.sort(rng.permutation(seen - keep_first)[:n - keep_first]) if n > keep_first else x[keep_first:]
            mixed = np.nonzero(rng.random(n) < 0.3)[0]
            mixed = mixed[mixed >= keep_first]
            x[mixed] = x[rng.permutation(mixed)]
        slot_pos[u, :n] = x
    p["state"].copy_(torch.from_numpy(st))
    if slot_pos.size:
        rows, there = _rows_of(p, ps, slot_pos.shape[1])
        p["pos"].view(-1)[rows[there]] = torch.from_numpy(slot_pos).cuda()[there]
    return p


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(c=c, scale=_scale(c))
    if c["op"] == "window":
        lens = _window_lens(c)
        rows = sum(lens) + 5                      # padding a batch is common
        s["start_host"] = _starts(lens)
        s["start"] = torch.from_numpy(s["start_host"]).cuda()
        s["q"] = _packed_tensor(gen, c["hq"], rows, c)
        s["k"] = _packed_tensor(gen, c["hkv"], rows, c)
        s["v"] = _packed_tensor(gen, c["hkv"], rows, c)
        s["o"] = torch.zeros_like(s["q"])
    else:
        lens = _unit_lens(c)
        if c["op"] == "append":
            new = _new_lens(c)
            s["start_host"] = _starts(new)
            rows = int(s["start_host"][-1]) + (5 if c["new"] > 1 else 0)
            s["k"] = _packed_tensor(gen, c["hkv"], rows, c)
            s["v"] = _packed_tensor(gen, c["hkv"], rows, c)
            s["w"] = torch.rand(c["hkv"], rows, generator=gen, device="cuda") if c["new"] > 1 else None
            s["cache"] = _pool(c, gen, seed, lens, lens + np.repeat(np.array(new, dtype=np.int64), c["hkv"]))
            s["state0"] = s["cache"]["state"].clone()
        else:
            s["cache"] = _pool(c, gen, seed, lens, lens)
            if c["op"] == "paged":
                s["q"] = _randn(gen, (c["batch"], c["hq"], c["d"]), c, 1.5)
                s["o"] = torch.zeros_like(s["q"])
                s["mass0"] = s["cache"]["mass"].clone()
            else:
                s["budget"] = torch.from_numpy(_budgets(c)).cuda()
                s["meta0"] = s["cache"]["meta"].clone()
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that uses the library keeps: parameters, workspace, cache handle."""
    from paper_2512_09238_b200 import binding as B
    c = s["c"]
    dt = B.TCA_BF16 if c["dtype"] == BF16 else B.TCA_F32
    s["prm"] = B.make_params(c.get("batch", c.get("n_seq")), c["hq"], c["hkv"], c["d"], 128, c.get("window", ALL),
                             sm_scale=s["scale"], dtype=dt)
    if c["op"] == "window":
        s["ws"] = B.alloc_workspace(s["prm"], s["q"].shape[1], B.TCA_OP_PACKED)
        return
    t = s["cache"]
    h = B.PagedCache(s["prm"], t["k"].shape[0], c["page"], t["table"].shape[1])
    for name in ("k", "v", "meta", "table"):
        getattr(h, name).copy_(t[name])
    s["handle"] = h
    s["cache"] = {name: getattr(h, name) for name in ("k", "v", "pos", "mass", "state", "table", "meta")}
    if c["op"] == "paged":
        s["ws"] = B.alloc_paged_workspace(s["prm"], h, c["mass"])


# ------------------------------------------------------------------ one pass
def run(state):
    s = state
    c = s["c"]
    op = c["op"]
    # every pass of a case begins with the cache as it was
    if op == "append":
        s["cache"]["state"].copy_(s["state0"])
    elif op == "evict":
        s["cache"]["meta"].copy_(s["meta0"])
    elif op == "paged" and c["mass"]:
        s["cache"]["mass"].copy_(s["mass0"])
    if own:
        from paper_2512_09238_b200 import binding as B
        if op == "window":
            B.tca_attn_window(s["prm"], s["q"], s["k"], s["v"], s["q"].shape[1], s["start"], c["n_sink"], s["o"], s["ws"])
            return s["o"]
        if op == "append":
            B.tca_paged_append(s["prm"], s["k"], s["v"], s["k"].shape[1], s["start_host"] if c["new"] > 1 else None, None,
                               s["w"], s["handle"])
            return _outputs(s["cache"])
        if op == "paged":
            B.tca_attn_paged(s["prm"], s["q"], s["handle"], c["n_sink"], c["mass"], s["o"], s["ws"])
            return (s["o"], s["cache"]["mass"]) if c["mass"] else s["o"]
        B.tca_paged_evict(s["prm"], s["handle"], c["n_sink"], c["n_recent"], s["budget"])
        return _outputs(s["cache"])
    if op == "window":
        return _plain_window(s)
    if op == "append":
        return _plain_append(s)
    if op == "paged":
        return _plain_paged(s)
    return _plain_evict(s)


def _outputs(t):
    return {name: t[name] for name in ("k", "v", "pos", "mass", "state")}


def _plain_window(s):
    """Sequence by sequence, in blocks of query rows against the sinks and the keys their windows reach."""
    c, o = s["c"], s["o"]
    H, G, d, w, sink = c["hkv"], c["hq"] // c["hkv"], c["d"], c["window"], c["n_sink"]
    step = 1024
    for lo, hi in zip(s["start_host"][:-1].tolist(), s["start_host"][1:].tolist()):
        for r0 in range(lo, hi, step):
            r1 = min(hi, r0 + step)
            first = max(lo, r0 - w + 1)
            sinks = min(sink, first - lo)
            key = torch.cat([torch.arange(lo, lo + sinks, device="cuda"), torch.arange(first, r1, device="cuda")])
            row = torch.arange(r0, r1, device="cuda")
            sees = (key[None] <= row[:, None]) & ((row[:, None] - key[None] < w) | (key[None] < lo + sink))
            q = s["q"][:, r0:r1].float().view(H, G, r1 - r0, d) * s["scale"]
            k, v = s["k"][:, key].float(), s["v"][:, key].float()
            x = q.reshape(H, G * (r1 - r0), d) @ k.transpose(-1, -2)
            x = x.view(H, G, r1 - r0, -1).masked_fill_(~sees, float("-inf"))
            x = x.sub_(x.amax(-1, keepdim=True)).exp_()
            total = x.sum(-1, keepdim=True)
            y = (x.view(H, G * (r1 - r0), -1) @ v).view(H, G, r1 - r0, d) / total
            o[:, r0:r1] = y.reshape(H * G, r1 - r0, d).to(o.dtype)
    return o


def _rows_of(t, ps, n):
    """Rows [U, n] of the flattened pool that hold every unit's slots, and which slots are in use."""
    j = torch.arange(n, device="cuda")
    there = j[None, :] < t["state"][:, :1]
    page = t["table"][:, :max(1, -(-n // ps))].long()
    rows = page[:, j // ps] * ps + j % ps if n else page[:, :0]
    return torch.where(there, rows, 0), there


def _plain_append(s):
    c, t = s["c"], s["cache"]
    H, ps = c["hkv"], c["page"]
    start = s["start_host"]
    new = np.diff(start)
    seq = np.repeat(np.arange(c["batch"]), new)
    i = torch.from_numpy(np.arange(start[-1]) - start[seq]).cuda()
    unit = torch.from_numpy(seq[None, :] * H + np.arange(H)[:, None]).cuda()            # [H, new rows]
    slot = t["state"][:, 0].long()[unit] + i
    dst = t["table"].long()[unit, slot // ps] * ps + slot % ps
    n = int(start[-1])
    t["k"].view(-1, c["d"])[dst] = s["k"][:, :n]
    t["v"].view(-1, c["d"])[dst] = s["v"][:, :n]
    t["pos"].view(-1)[dst] = (t["state"][:, 1].long()[unit] + i).int()
    t["mass"].view(-1)[dst] = s["w"][:, :n] if s["w"] is not None else torch.zeros((), device="cuda")
    t["state"][:, :2] += torch.from_numpy(np.repeat(new, H).astype(np.int32)).cuda()[:, None]
    return _outputs(t)


def _plain_paged(s):
    c, t = s["c"], s["cache"]
    B, H, G, d = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["d"]
    n = min(c["ctx"], t["table"].shape[1] * c["page"])       # no unit is longer
    rows, there = _rows_of(t, c["page"], n)
    lens = t["state"][:, :1].long()
    j = torch.arange(n, device="cuda")[None, :]
    there = there & ((j >= lens - c["window"]) | (j < c["n_sink"]))
    q = s["q"].float().view(B * H, G, d) * s["scale"]
    k = t["k"].view(-1, d)[rows].float()
    x = (q @ k.transpose(-1, -2)).masked_fill_(~there[:, None, :], float("-inf"))
    del k
    top = x.amax(-1, keepdim=True)
    x = (x - torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    v = t["v"].view(-1, d)[rows].float().masked_fill_(~there[:, :, None], 0.0)
    out = torch.where(total > 0, (x @ v) / total, 0.0)
    s["o"].copy_(out.view(B, c["hq"], d))
    if not c["mass"]:
        return s["o"]
    share = (x / total).mean(1)
    t["mass"].view(-1)[rows[there]] += share[there]
    return s["o"], t["mass"]


def _plain_evict(s):
    c, t = s["c"], s["cache"]
    n = min(c["ctx"], t["table"].shape[1] * c["page"])       # no unit is longer
    rows, there = _rows_of(t, c["page"], n)
    lens, budget = t["state"][:, 0].long(), s["budget"].long()
    j = torch.arange(n, device="cuda")[None, :]
    pos = torch.where(there, t["pos"].view(-1)[rows].long(), -1)
    safe = there & ((j < c["n_sink"]) | (pos > pos.amax(1, keepdim=True) - c["n_recent"]))
    # safe rows first, then by mass, then what is not there; equal ones by slot
    key = t["mass"].view(-1)[rows].double().masked_fill(safe, math.inf).masked_fill(~there, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(1, order, j.expand_as(order).contiguous())
    over = (lens > budget)[:, None]
    kept = there & (rank < budget[:, None])
    hole = over & ~kept & (j < budget[:, None])
    late = over & kept & (j >= budget[:, None])
    dst, src = rows[hole], rows[late]          # unit after unit, ascending slots: as many of one as of the other
    for name in ("k", "v"):
        x = t[name].view(-1, c["d"])
        x[dst] = x[src]
    for name in ("pos", "mass"):
        x = t[name].view(-1)
        x[dst] = x[src]
    t["state"][:, 0] = torch.minimum(lens, budget).int()
    return _outputs(t)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    e, d = 2 if c["dtype"] == BF16 else 4, c["d"]
    G = c["hq"] // c["hkv"]
    if c["op"] == "window":
        rows = pairs = 0
        w, sink = c["window"], c["n_sink"]
        for n in _window_lens(c):
            i = np.arange(n, dtype=np.int64)
            pairs += int((np.minimum(i + 1, w) + np.minimum(sink, np.maximum(0, i + 1 - w))).sum())
            rows += n
        return dict(bytes=rows * d * e * (2 * c["hq"] + 2 * c["hkv"]), flops=4 * d * c["hq"] * pairs)
    lens = _unit_lens(c)
    if c["op"] == "append":
        rows = sum(_new_lens(c)) * c["hkv"]
        return dict(bytes=rows * (4 * d * e + 8 + (4 if c["new"] > 1 else 0)), flops=0)
    if c["op"] == "paged":
        s, lo = _visible(c, lens)
        rows = int((s + lens - lo).sum())
        return dict(bytes=rows * (2 * d * e + (8 if c["mass"] else 0)) + 2 * c["batch"] * c["hq"] * d * e,
                    flops=4 * d * G * rows)
    # rows move from behind the budget to the holes in front of it: what is kept at random, and what is recent or not
    budget = _budgets(c).astype(np.float64)
    over = lens > budget
    moved = np.where(over, (lens - budget) * budget / np.maximum(1, lens), 0.0).sum()
    return dict(bytes=int(8 * lens[over].sum() + moved * 2 * (2 * d * e + 8)), flops=0)


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    c = dict(case)
    global own
    keep_own, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = keep_own
    G, d, scale, H = c["hq"] // c["hkv"], c["d"], s["scale"], c["hkv"]
    if c["op"] == "window":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lo = 0
        for n in _window_lens(c):
            k, v = s["k"][:, lo:lo + n].double(), s["v"][:, lo:lo + n].double()
            for a in range(0, n, 2048):
                b = min(n, a + 2048)
                i = torch.arange(a, b, device="cuda")[:, None]
                near = max(0, a - c["window"] + 1)
                j = torch.arange(near, b, device="cuda")
                far = torch.arange(min(c["n_sink"], near), device="cuda")
                j = torch.cat([far, j])[None, :]
                hidden = (j > i) | ((j <= i - c["window"]) & (j >= c["n_sink"]))
                for h in range(c["hq"]):
                    x = (s["q"][h, lo + a:lo + b].double() @ k[h // G][j[0]].T) * scale
                    out[h, lo + a:lo + b] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v[h // G][j[0]]
            lo += n
        return out
    t, ps = s["cache"], c["page"]
    table = t["table"].cpu().numpy().astype(np.int64)
    lens = _unit_lens(c)

    def at(u, slots):
        return torch.from_numpy(table[u, slots // ps] * ps + slots % ps).cuda()

    if c["op"] == "paged":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        mass = t["mass"].double().view(-1)
        for u in range(len(lens)):
            n = int(lens[u])
            slots = np.array([x for x in (range(n) if c["window"] >= n else
                                          sorted(set(range(min(n, c["n_sink"]))) | set(range(n - c["window"], n))))], dtype=np.int64)
            if len(slots) == 0:
                continue
            r = at(u, slots)
            b, h = u // H, u % H
            p = torch.softmax(s["q"][b, h * G:(h + 1) * G].double() @ t["k"].view(-1, d)[r].double().T * scale, -1)
            out[b, h * G:(h + 1) * G] = p @ t["v"].view(-1, d)[r].double()
            mass[r] += p.mean(0)
        return (out, mass.view(t["mass"].shape)) if c["mass"] else out
    k, v, mass = t["k"].double().view(-1, d), t["v"].double().view(-1, d), t["mass"].double().view(-1)
    if c["op"] == "append":
        lo = 0
        for b, n in enumerate(_new_lens(c)):
            for h in range(H if n else 0):
                u = b * H + h
                r = at(u, int(lens[u]) + np.arange(n))
                k[r], v[r] = s["k"][h, lo:lo + n].double(), s["v"][h, lo:lo + n].double()
                mass[r] = s["w"][h, lo:lo + n].double() if s["w"] is not None else 0.0
            lo += n
    else:
        budgets = _budgets(c)
        for u in range(len(lens)):
            n, budget = int(lens[u]), int(budgets[u])
            if n <= budget:
                continue
            r = at(u, np.arange(n))
            m, pos = mass[r].cpu().numpy(), t["pos"].view(-1)[r].cpu().numpy()
            slot = np.arange(n)
            must = (slot < c["n_sink"]) | (pos > pos.max() - c["n_recent"])
            free = slot[~must]
            best = free[np.lexsort((free, -m[free]))]
            kept = must.copy()
            kept[best[:budget - int(must.sum())]] = True
            holes, late = slot[:budget][~kept[:budget]], slot[budget:][kept[budget:]]
            for x in (k, v, mass):
                x[r[torch.from_numpy(holes).cuda()]] = x[r[torch.from_numpy(late).cuda()]]
    return dict(k=k.view(t["k"].shape), v=v.view(t["v"].shape), pos=None, mass=mass.view(t["mass"].shape), state=None)
