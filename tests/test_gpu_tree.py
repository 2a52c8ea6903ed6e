"""tca_attn_tree and tca_cache_accept against the oracle and against one append per token."""
import numpy as np
import pytest
import torch

import serving_harness as H
from paper_2512_09238_b200 import binding as B

pytestmark = pytest.mark.gpu


def drafts(prm, T, dtype, seed):
    b, d = prm.batch, prm.head_dim
    return (H.randn(seed, (b, prm.n_q_heads, T, d), dtype, 1.5), H.randn(seed + 1, (b, prm.n_kv_heads, T, d), dtype),
            H.randn(seed + 2, (b, prm.n_kv_heads, T, d), dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 2, 5, 16, 33, 64, 127, 128])
def test_drafted_counts(T, d, dtype):
    prm = H.params(2, 4, 2, d, dtype)
    cache = H.make_cache(prm, [300, 0, 17, 128], [70, 95, 1, 64], [90, 3, 50, 0], 500, dtype, 1)   # the first ring wraps
    q, kd, vd = drafts(prm, T, dtype, 10)
    parent = np.stack([H.chain(T), H.bush(T, 3)])
    H.check_tree(prm, q, kd, vd, parent, cache, H.run_tree(prm, q, kd, vd, parent, cache), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8])
def test_groups(group, dtype):
    prm = H.params(1, 2 * group, 2, 128, dtype)
    cache = H.make_cache(prm, [260, 40], [90, 20], [30, 90], 400, dtype, 2)
    q, kd, vd = drafts(prm, 37, dtype, 20)
    parent = H.bush(37, 5)[None]
    H.check_tree(prm, q, kd, vd, parent, cache, H.run_tree(prm, q, kd, vd, parent, cache), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_empty_caches_and_live_counts(dtype):
    """Units without a row (all, and some), and sequences that drafted fewer tokens or none."""
    prm = H.params(3, 4, 2, 128, dtype)
    T, live = 9, np.array([9, 0, 4])
    q, kd, vd = drafts(prm, T, dtype, 30)
    parent = np.stack([H.bush(T, i) for i in range(3)])
    for n_global, n_tail in ((0, 0), ([0, 5, 0, 0, 400, 0], [0, 0, 0, 3, 96, 0])):
        cache = H.make_cache(prm, n_global, n_tail, 0, 500, dtype, 3, tail_cap=97)
        for x in (q, kd, vd):                                # what is not drafted is not used
            x[1], x[2, :, 4:] = float("nan"), float("nan")
        H.check_tree(prm, q, kd, vd, parent, cache, H.run_tree(prm, q, kd, vd, parent, cache, n_live=live), dtype, n_live=live)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_units_than_registers_hold_and_uneven_ones(dtype):
    """150 units (more than are kept in registers), lengths from 0 to 700."""
    prm = H.params(50, 3, 3, 64, dtype)
    r = np.random.default_rng(4)
    ng, nt = r.integers(0, 600, 150), r.integers(0, 96, 150)
    ng[::7], nt[::7] = 0, 0
    cache = H.make_cache(prm, ng, nt, r.integers(0, 96, 150), 800, dtype, 6)
    q, kd, vd = drafts(prm, 3, dtype, 40)
    parent = np.tile(H.chain(3), (50, 1))
    H.check_tree(prm, q, kd, vd, parent, cache, H.run_tree(prm, q, kd, vd, parent, cache), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_cache(dtype):
    prm = H.params(1, 8, 2, 128, dtype, block=128, window=1024)
    cache = H.make_cache(prm, [9000, 2500], [1100, 1024], [1000, 0], 40000, dtype, 7)
    q, kd, vd = drafts(prm, 24, dtype, 50)
    parent = H.bush(24, 9)[None]
    got = H.run_tree(prm, q, kd, vd, parent, cache)
    H.check_tree(prm, q, kd, vd, parent, cache, got, dtype, heads=(0, 5))
    assert torch.equal(got, H.run_tree(prm, q, kd, vd, parent, cache))            # the same bits every time
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        again = H.run_tree(prm, q, kd, vd, parent, cache)
    torch.cuda.synchronize()
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_a_row_does_not_see_has_no_influence(bad, dtype):
    """Other branches, cache rows not in use, and the other sequence's cache may hold anything."""
    prm = H.params(2, 4, 2, 128, dtype)
    cache = H.make_cache(prm, [70, 300, 129, 1], [90, 30, 96, 20], [50, 0, 20, 90], 500, dtype, 8, extra_cap=40, tail_cap=97)
    T = 12
    q, kd, vd = drafts(prm, T, dtype, 60)
    parent = np.stack([H.chain(T), np.array([-1, -1, 0, 1, 2, 3, 0, 6, 5, -1, 4, 7], dtype=np.int32)])
    clean = H.run_tree(prm, q, kd, vd, parent, cache)
    used = np.zeros(cache.rows_total, dtype=bool)
    for u in (2, 3):
        used[cache.unit_rows(u)] = True
    hide = torch.from_numpy(~used).cuda()
    cache.k[hide], cache.v[hide] = bad, bad                   # everything but the second sequence's rows
    kd[1, :, 3], vd[1, :, 3] = bad, bad                       # seen by 3, 5 and 8 only
    got = H.run_tree(prm, q, kd, vd, parent, cache)
    clear = [t for t in range(T) if t not in (3, 5, 8)]
    assert torch.equal(got[1][:, clear], clean[1][:, clear])
    assert not torch.isfinite(got[1][:, [3, 5, 8]].float()).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 3, 5, 7, 8])
def test_a_drafted_token_rounds_the_same_whatever_shares_its_tile(group, dtype):
    """Bit for bit, while the other drafted tokens, those past n_live and the calls before hold large queries."""
    prm = H.params(2, 2 * group, 2, 128, dtype)
    cache = H.make_cache(prm, [700, 90, 260, 1500], [90, 30, 96, 20], [50, 0, 20, 90], 2000, dtype, 12)
    T, live = 21, np.array([21, 13])
    q, kd, vd = drafts(prm, T, dtype, 64)
    q *= 3
    parent = np.stack([H.bush(T, 3), H.chain(T)])
    first = H.run_tree(prm, q, kd, vd, parent, cache, n_live=live)
    for quiet in ([0], [1, 2, 7], list(range(10)), list(range(13))):
        loud = q * 50
        H.run_tree(prm, loud, kd, vd, parent, cache)
        loud[:, :, quiet] = q[:, :, quiet]
        got = H.run_tree(prm, loud, kd, vd, parent, cache, n_live=live)
        assert torch.equal(got[:, :, quiet], first[:, :, quiet])


@pytest.mark.parametrize("flags", [0, B.TCA_FLAG_PREFILL_SIMT])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [2, 70])
def test_nan_keys_that_are_seen_show(T, dtype, flags):
    """A unit whose cached keys are all NaN (so that no partial result has a maximum), and one with a single NaN."""
    prm = H.params(1, 6, 3, 128, dtype, flags=flags)
    cache = H.make_cache(prm, [700, 300, 2], [0, 50, 1], 0, 900, dtype, 13)
    q, kd, vd = drafts(prm, T, dtype, 67)
    parent = H.chain(T)[None]
    clean = H.run_tree(prm, q, kd, vd, parent, cache)
    cache.k[torch.from_numpy(cache.unit_rows(0)).cuda()] = float("nan")
    cache.k[int(cache.unit_rows(2)[1]), 7] = float("nan")
    got = H.run_tree(prm, q, kd, vd, parent, cache)
    assert torch.isnan(got[:, [0, 1, 4, 5]]).all()
    assert torch.equal(got[:, 2:4], clean[:, 2:4])


def test_parents_that_do_not_precede_their_child_count_as_roots():
    prm = H.params(1, 2, 1, 64, "bf16")
    cache = H.make_cache(prm, 20, 30, 0, 50, "bf16", 9)
    q, kd, vd = drafts(prm, 6, "bf16", 70)
    odd = np.array([[0, 5, -9, 1, 2, 1 << 30]], dtype=np.int32)
    root = np.array([[-1, -1, -1, 1, 2, -1]], dtype=np.int32)
    if B.tca_build_info() == 0:
        assert torch.equal(H.run_tree(prm, q, kd, vd, odd, cache), H.run_tree(prm, q, kd, vd, root, cache))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_drafted_token_equals_append_and_decode(dtype):
    prm = H.params(2, 8, 2, 128, dtype)
    cache = H.make_cache(prm, [200, 31, 0, 64], 60, 10, 300, dtype, 11, extra_cap=8)
    q, kd, vd = drafts(prm, 1, dtype, 80)
    parent = np.full((2, 1), -1, dtype=np.int32)
    got = H.run_tree(prm, q, kd, vd, parent, cache)
    H.check_tree(prm, q, kd, vd, parent, cache, got, dtype)
    B.tca_cache_append(prm, cache, kd[:, :, 0].contiguous(), vd[:, :, 0].contiguous(), q[:, :, 0].contiguous())
    out = torch.empty_like(q[:, :, 0]).contiguous()
    B.tca_attn_decode(prm, q[:, :, 0].contiguous(), cache, out, B.alloc_workspace(prm, cache.rows_total, B.TCA_OP_DECODE))
    diff = (out.float() - got[:, :, 0].float()).abs().max().item()
    # each side is within half a bf16 step of P and of the result (values of size 1), or fp32 rounding
    assert diff <= (2 * 2 * 2.0 ** -8 * 4 if dtype == "bf16" else 1e-4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_call_replays_over_a_cache_that_has_grown(dtype):
    prm = H.params(1, 4, 2, 128, dtype, block=32, window=64)
    cache = H.make_cache(prm, [3, 200], [20, 90], 0, 300, dtype, 12, extra_cap=2000, t_keep=32)
    T = 8
    q, kd, vd = drafts(prm, T, dtype, 90)
    parent = H.bush(T, 2)[None]
    par = torch.from_numpy(parent).cuda()
    ws, o = B.alloc_tree_workspace(prm, T), torch.zeros_like(q)
    B.tca_attn_tree(prm, q, kd, vd, T, par, None, cache, o, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.tca_attn_tree(prm, q, kd, vd, T, par, None, cache, o, ws)
    path = torch.arange(T, dtype=torch.int32, device="cuda")[None].contiguous()
    for step in range(60):
        B.tca_cache_accept(prm, cache, kd, vd, q, T, path, np.array([T], dtype=np.int32))
        if step in (0, 20, 59):
            g.replay()
            torch.cuda.synchronize()
            assert B.tca_ws_status(ws) == B.TCA_OK
            H.check_tree(prm, q, kd, vd, parent, cache, o, dtype)


@pytest.mark.parametrize("T", [3, 40, 128])
def test_tensor_cores_agree_with_the_fp32_pipes(T):
    cache_of = lambda p: H.make_cache(p, [700, 130], [90, 64], 40, 900, "bf16", 19)  # noqa: E731
    prm, simt = H.params(1, 8, 2, 128, "bf16"), H.params(1, 8, 2, 128, "bf16", flags=B.TCA_FLAG_PREFILL_SIMT)
    cache = cache_of(prm)
    q, kd, vd = drafts(prm, T, "bf16", 160)
    parent = H.bush(T, 1)[None]
    for p in (prm, simt):
        H.check_tree(p, q, kd, vd, parent, cache, H.run_tree(p, q, kd, vd, parent, cache), "bf16", heads=(0, 5))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_into_a_large_cache(dtype):
    """A unit whose rows lie more than 2^31 elements into the cache: attended to, and appended to."""
    d, far, T = 128, (1 << 31) // 128 + 1000, 6
    prm = H.params(2, 2, 1, d, dtype, block=32, window=64)
    cache = B.Cache(prm, np.array([far, 256]), 96, np.full(2, 8), init=False)
    cache.n_global[:], cache.n_tail[:], cache.tail_head[:], cache.seq_len[:] = [0, 200], [3, 94], [0, 50], [3, 400]
    B.tca_cache_init(prm, cache)
    for u in range(2):
        rows = torch.from_numpy(cache.unit_rows(u)).cuda()
        cache.k[rows], cache.v[rows] = H.randn(u, (len(rows), d), dtype), H.randn(9 + u, (len(rows), d), dtype)
        cache.pos[rows] = torch.arange(len(rows), dtype=torch.int32, device="cuda")
    q, kd, vd = drafts(prm, T, dtype, 170)
    parent = np.stack([H.chain(T), H.bush(T, 4)])
    H.check_tree_rows(prm, q, kd, vd, parent, cache, H.run_tree(prm, q, kd, vd, parent, cache), dtype)
    path = torch.arange(T, dtype=torch.int32, device="cuda").repeat(2, 1)
    ng, nt, sl = int(cache.n_global[1]), int(cache.n_tail[1]), int(cache.seq_len[1])
    B.tca_cache_accept(prm, cache, kd, vd, q, T, path, np.array([2, T], dtype=np.int32))      # the second compresses
    torch.cuda.synchronize()
    H.mirror_equals_device(cache)
    assert (cache.n_global[1], cache.n_tail[1], cache.seq_len[1]) == (ng + 8, nt + T - 32, sl + T)
    rows = torch.from_numpy(cache.unit_rows(1)).cuda()[-T:]
    assert torch.equal(cache.k[rows], kd[1, 0]) and torch.equal(cache.v[rows], vd[1, 0])
    assert cache.pos[rows].tolist() == list(range(sl, sl + T))


def test_a_set_status_word_stops_the_call():
    prm = H.params(1, 4, 2, 128, "bf16")
    cache = H.make_cache(prm, 200, 90, 0, 300, "bf16", 17)
    q, kd, vd = drafts(prm, 5, "bf16", 140)
    par = torch.from_numpy(H.chain(5)[None].copy()).cuda()
    ws, o = B.alloc_tree_workspace(prm, 5), torch.full_like(q, 7.0)
    ws[:4] = torch.tensor([1, 0, 0, 0], dtype=torch.uint8, device="cuda")
    B.tca_attn_tree(prm, q, kd, vd, 5, par, None, cache, o, ws)
    assert B.tca_ws_status(ws) == B.TCA_ERR_TIMEOUT and (o == 7.0).all()
    ws.zero_()
    H.check_tree(prm, q, kd, vd, H.chain(5)[None], cache, H.run_tree(prm, q, kd, vd, H.chain(5)[None], cache, ws=ws), "bf16")


def test_one_workspace_serves_calls_of_different_shapes():
    """A workspace sized for the largest call holds what earlier, larger calls left behind."""
    prm = H.params(3, 8, 2, 128, "bf16")
    cache = H.make_cache(prm, [900, 5, 0, 300, 260, 40], [90, 3, 0, 64, 10, 95], 20, 1000, "bf16", 18)
    ws = B.alloc_tree_workspace(prm, 100)
    for T in (100, 3, 32, 1, 65):
        q, kd, vd = drafts(prm, T, "bf16", 150 + T)
        parent = np.stack([H.bush(T, T + i) for i in range(3)])
        H.check_tree(prm, q, kd, vd, parent, cache, H.run_tree(prm, q, kd, vd, parent, cache, ws=ws), "bf16", heads=(0, 7))


# ------------------------------------------------------------------ tca_cache_accept
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block,window,n_tail,T", [(32, 64, 60, 20), (32, 64, 95, 9), (16, 8, 23, 64), (1, 1, 1, 12),
                                                   (1, 0, 0, 5), (128, 0, 100, 128), (8, 40, 47, 33)])
def test_accept_equals_one_append_per_token(block, window, n_tail, T, dtype):
    """Bit for bit, for sequences that accept different numbers of tokens (none, one, all)."""
    prm = H.params(5, 6, 2, 64, dtype, block=block, window=window)
    cache = H.make_cache(prm, 20, min(n_tail, window + block - 1), (window + block) // 2, 400, dtype, 13,
                         t_keep=max(1, block // 3), extra_cap=2 * T + 200)
    q, kd, vd = drafts(prm, T, dtype, 100)
    r = np.random.default_rng(T)
    n = np.array([0, 1, T, max(1, T // 2), max(1, T - 1)], dtype=np.int32)
    path = np.stack([np.sort(r.permutation(T)) if s != 3 else r.permutation(T) for s in range(5)]).astype(np.int32)
    ref = H.clone_cache(prm, cache)
    B.tca_cache_accept(prm, cache, kd, vd, q, T, torch.from_numpy(path).cuda(), n)
    torch.cuda.synchronize()
    H.mirror_equals_device(cache)
    assert B.tca_cache_status(cache)[0] == B.TCA_OK
    for step in range(T + 1):
        for s in range(5):
            if n[s] != step:
                continue
            for u in (2 * s, 2 * s + 1):
                lo = int(cache.seg_start[u])
                seg = slice(lo, lo + int(cache.global_cap[u]) + cache.tail_cap)
                for name in ("k", "v", "pos"):
                    assert torch.equal(getattr(cache, name)[seg], getattr(ref, name)[seg]), (name, s)
                w = slice(u * B.TCA_STATE_WORDS, (u + 1) * B.TCA_STATE_WORDS)
                assert torch.equal(cache.state[w], ref.state[w])
        if step < T:
            tok = [int(path[s][step]) for s in range(5)]
            pick = lambda x: torch.stack([x[s, :, tok[s]] for s in range(5)]).contiguous()  # noqa: E731
            B.tca_cache_append(prm, ref, pick(kd), pick(vd), pick(q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("block,t_keep", [(1, 1), (2, 1), (8, 3), (32, 31), (64, 20), (128, 41), (128, 128)])
def test_a_block_that_leaves_keeps_what_the_formula_says(block, t_keep, group, d, dtype):
    """The kept positions against fp64, for keys that are all different, repeated (equal scores go to the earlier
    position) and all the same."""
    hkv, window = 3, 5
    prm = H.params(1, group * hkv, hkv, d, dtype, block=block, window=window)
    full = window + block
    cache = H.make_cache(prm, 9, full - 1, full // 3, 500, dtype, 18, t_keep=t_keep, extra_cap=t_keep + 2)
    q, kd, vd = drafts(prm, 2, dtype, 140)
    rows = [cache.unit_rows(u)[9:9 + min(block, full - 1)] for u in range(hkv)]
    r = np.random.default_rng(block + group)
    cache.k[torch.from_numpy(rows[1]).cuda()] = cache.k[torch.from_numpy(r.choice(rows[1][:5], len(rows[1]))).cuda()]
    cache.k[torch.from_numpy(rows[2]).cuda()] = cache.k[int(rows[2][0])].clone()
    keys, first = [H.f64(cache.k[torch.from_numpy(x).cuda()]) for x in rows], 500 - (full - 1)
    B.tca_cache_accept(prm, cache, kd, vd, q, 2, torch.ones(1, 2, dtype=torch.int32, device="cuda"), np.array([1], dtype=np.int32))
    H.mirror_equals_device(cache)
    pos, kk = cache.pos.cpu().numpy(), H.f64(cache.k)
    for u in range(hkv):
        x = H.f64(q)[0, u * group:(u + 1) * group, 1] @ keys[u].T * H.scale_of(d)
        score = np.log(np.mean(np.exp(x - np.log(np.exp(x - x.max(1, keepdims=True)).sum(1, keepdims=True)) - x.max(1, keepdims=True)), axis=0))
        # equal keys have equal scores; different ones differ by far more than fp64 rounds
        kept = np.sort(np.lexsort((np.arange(len(score)), -np.round(score, 9)))[:t_keep])
        lo = int(cache.seg_start[u]) + 9
        assert np.array_equal(pos[lo:lo + t_keep], first + kept), u
        assert np.array_equal(kk[lo:lo + t_keep], keys[u][kept]), u


def test_accept_of_more_sequences_than_one_launch_takes():
    batch, T = 1500, 2
    prm = H.params(batch, 1, 1, 64, "bf16", block=8, window=8)
    r = np.random.default_rng(3)
    cache = H.make_cache(prm, 4, 0, 0, 40, "bf16", 19, t_keep=2, extra_cap=4, tail_cap=17)
    cache.n_tail[:] = r.integers(3, 16, batch)
    cache.seq_len[:] = 30 + cache.n_tail
    B.tca_cache_init(prm, cache)
    q, kd, vd = drafts(prm, T, "bf16", 150)
    n = (r.random(batch) < 0.6).astype(np.int32)
    n[1020:1030] = 1
    path = r.integers(0, T, (batch, T)).astype(np.int32)
    before, ref = H.clone_cache(prm, cache), H.clone_cache(prm, cache)
    pick = lambda x: x[torch.arange(batch), :, torch.from_numpy(path[:, 0]).long()].contiguous()  # noqa: E731
    B.tca_cache_append(prm, ref, pick(kd), pick(vd), pick(q))
    B.tca_cache_accept(prm, cache, kd, vd, q, T, torch.from_numpy(path).cuda(), n)
    H.mirror_equals_device(cache)
    took = torch.from_numpy(n > 0).cuda()
    per_unit = cache.rows_total // batch
    for name in ("k", "v", "pos"):
        a, b, c = (getattr(x, name).view(batch, per_unit, -1) for x in (cache, ref, before))
        assert torch.equal(a, torch.where(took[:, None, None], b, c)), name


def test_accept_takes_the_same_token_twice_and_clamps_the_path():
    prm = H.params(1, 2, 1, 64, "bf16", block=32, window=64)
    q, kd, vd = drafts(prm, 4, "bf16", 110)
    a = H.make_cache(prm, 5, 10, 0, 15, "bf16", 14)
    b = H.clone_cache(prm, a)
    n = np.array([3], dtype=np.int32)
    B.tca_cache_accept(prm, a, kd, vd, q, 4, torch.tensor([[2, 2, 3, 0]], dtype=torch.int32, device="cuda"), n)
    if B.tca_build_info() == 0:
        B.tca_cache_accept(prm, b, kd, vd, q, 4, torch.tensor([[2, 2, 99, -1]], dtype=torch.int32, device="cuda"), n)
        torch.cuda.synchronize()
        assert torch.equal(a.k, b.k) and torch.equal(a.pos, b.pos)


def test_accept_refuses_without_touching_anything():
    prm = H.params(2, 2, 1, 64, "bf16", block=32, window=64)
    q, kd, vd = drafts(prm, 8, "bf16", 120)
    cache = H.make_cache(prm, [5, 6], [92, 10], 0, 100, "bf16", 15, extra_cap=0)
    before = H.clone_cache(prm, cache)
    path = torch.zeros(2, 8, dtype=torch.int32, device="cuda")
    for n, status in (([4, 0], B.TCA_ERR_CAPACITY), ([9, 0], B.TCA_ERR_INVALID_ARG), ([-1, 0], B.TCA_ERR_INVALID_ARG)):
        with pytest.raises(B.TcaError) as e:
            B.tca_cache_accept(prm, cache, kd, vd, q, 8, path, np.array(n, dtype=np.int32))
        assert e.value.status == status
    torch.cuda.synchronize()
    for name in ("k", "v", "pos", "state"):
        assert torch.equal(getattr(cache, name), getattr(before, name))
    H.mirror_equals_device(cache)
    B.tca_cache_accept(prm, cache, kd, vd, q, 8, path, np.array([3, 8], dtype=np.int32))    # what fits is taken


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("call", ["accept", "append"])
def test_a_replayed_call_without_room_leaves_the_unit_as_it_was(call, dtype):
    """A captured accept or append moves the device state on at every replay. Units that run out of room stop there,
    each as its last call with room left it; the others go on, and nothing outside their segments is written."""
    T = 40 if call == "accept" else 1
    prm = H.params(3, 4, 2, 64, dtype, block=8, window=16)
    cache = H.make_cache(prm, 3, 20, 5, 60, dtype, 23, t_keep=3, extra_cap=[0, 20, 16, 47, 0, 31])
    q, kd, vd = drafts(prm, T, dtype, 180)
    ref = H.clone_cache(prm, cache)
    full, n = 24, np.array([T, T - 1 if T > 1 else 1, 0 if T > 1 else 1], dtype=np.int32)
    path = torch.arange(T, dtype=torch.int32, device="cuda").repeat(3, 1)
    one = [x[:, :, 0].contiguous() for x in (kd, vd, q)]

    def run(c, n=n):
        if call == "accept":
            B.tca_cache_accept(prm, c, kd, vd, q, T, path, n)
        else:
            B.tca_cache_append(prm, c, *one)

    # the mirror allows one call for all units; made ready once so that the capture sees no first-call work
    warm = H.make_cache(prm, 3, 20, 5, 60, dtype, 23, t_keep=3, extra_cap=600)
    run(warm)
    torch.cuda.synchronize()
    if call == "accept":
        n[0] = 3                      # unit 0 has no room for a block: few enough tokens at first, too many on replay
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(cache, n)
    # what each unit's replays do, by the counts: it takes the call's tokens while there is room for their blocks
    room, tail, glob, seq = (x.copy() for x in (ref.global_cap, ref.n_tail, ref.n_global, ref.seq_len))
    taken = np.zeros(6, dtype=int)
    replays = 30 if call == "accept" else 200
    for _ in range(replays):
        for u in range(6):
            k = int(n[u // 2])
            over = tail[u] + k - full
            blocks = over // 8 + 1 if over >= 0 else 0
            if k and glob[u] + 3 * blocks <= room[u]:
                taken[u] += 1
                tail[u], glob[u], seq[u] = tail[u] + k - 8 * blocks, glob[u] + 3 * blocks, seq[u] + k
        g.replay()
    torch.cuda.synchronize()
    st = cache.state.view(6, -1).cpu().numpy()
    assert np.array_equal(st[:, 2], glob) and np.array_equal(st[:, 4], tail) and np.array_equal(st[:, 5], seq)
    assert 0 < taken.max() < replays
    status, detail = B.tca_cache_status(cache)
    stopped = [u for u in range(6) if n[u // 2] and taken[u] < replays]
    assert status == B.TCA_ERR_BOUNDS and list(detail) == [stopped[0], 5, glob[stopped[0]]]
    # the same numbers of tokens without a graph, in a cache with room, unit by unit
    wide = H.make_cache(prm, 3, 20, 5, 60, dtype, 23, t_keep=3, extra_cap=600)
    for u in range(6):
        a, b = int(wide.seg_start[u]), int(ref.seg_start[u])
        for name in ("k", "v", "pos"):
            src, dst = getattr(ref, name), getattr(wide, name)
            dst[a:a + 3] = src[b:b + 3]
            dst[a + int(wide.global_cap[u]):a + int(wide.global_cap[u]) + 24] = src[b + int(ref.global_cap[u]):b + int(ref.global_cap[u]) + 24]
    for step in range(int(taken.max()) + 1):
        for u in range(6):
            if taken[u] != step or n[u // 2] == 0:
                continue
            ng, a, b = int(glob[u]), int(wide.seg_start[u]), int(cache.seg_start[u])
            for name in ("k", "v", "pos"):
                x, y = getattr(wide, name), getattr(cache, name)
                assert torch.equal(x[a:a + ng], y[b:b + ng]), (name, u)
                slots = (int(st[u, 3]) + torch.arange(int(tail[u]), device="cuda")) % 24
                assert torch.equal(x[a + int(wide.global_cap[u]) + slots], y[b + int(cache.global_cap[u]) + slots]), (name, u)
                left = slice(b + ng, b + int(cache.global_cap[u]))          # free rows of the global region
                assert torch.equal(y[left], getattr(ref, name)[left]), (name, u)
        if step < taken.max():
            run(wide, n)
    # and a call by the mirror, which has not moved, is stopped by the unit's own words too
    before = cache.state.clone()
    if call == "append":
        run(cache)
        torch.cuda.synchronize()
        assert torch.equal(cache.state.view(6, -1)[stopped], before.view(6, -1)[stopped])


# ------------------------------------------------------------------ the operators together
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_to_drafted_tokens_as_a_server_runs_them(dtype):
    """Packed prompts -> attention -> cache -> drafted tree -> accepted path -> decode; a prompt joins later."""
    from oracle import serving_oracle as S
    hq, hkv, d, T = 4, 2, 128, 7
    lens = [210, 33, 150]
    prm4 = H.params(4, hq, hkv, d, dtype, block=32, window=64)
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    q, k, v = (H.packed_buffer(200 + i, h, int(starts[-1]), d, dtype, "tokens") for i, h in enumerate((hq, hkv, hkv)))
    o = H.run_packed(H.params(3, hq, hkv, d, dtype), q, k, v, starts)
    want, a, s = S.packed_attention(H.f64(q), H.f64(k), H.f64(v), starts, H.scale_of(d))
    H.check(H.f64(o), want, S.attention_tolerance(want, a, s, d, np.full(want.shape[:2], 210), dtype), "prompts")
    cache = B.Cache(prm4, np.full(8, 256, dtype=np.int64), 96, np.full(8, 8, dtype=np.int64))
    B.tca_cache_load(prm4, k, v, int(starts[-1]), starts, np.array([2, 0, 3], dtype=np.int32), cache)
    ws = B.alloc_tree_workspace(prm4, T)
    dec_ws = B.alloc_workspace(prm4, cache.rows_total, B.TCA_OP_DECODE)
    for step in range(6):
        qd, kd, vd = drafts(prm4, T, dtype, 300 + 10 * step)
        parent = np.stack([H.bush(T, step + i) for i in range(4)])
        live = np.array([T, 0 if step < 3 else T, T, 3], dtype=np.int32)
        got = H.run_tree(prm4, qd, kd, vd, parent, cache, n_live=live, ws=ws)
        H.check_tree(prm4, qd, kd, vd, parent, cache, got, dtype, n_live=live)
        n = np.minimum(live, [3, 2, 5, 1]).astype(np.int32)
        path = torch.from_numpy(np.tile(np.arange(T, dtype=np.int32), (4, 1))).cuda()
        B.tca_cache_accept(prm4, cache, kd, vd, qd, T, path, n)
        H.mirror_equals_device(cache)
        if step == 2:      # the idle slot gets its prompt while the others go on
            B.tca_cache_load(prm4, k, v, int(starts[-1]), starts[1:3].copy(), np.array([1], dtype=np.int32), cache)
    qn = H.randn(999, (4, hq, d), dtype, 1.5)
    out = torch.empty_like(qn)
    B.tca_attn_decode(prm4, qn, cache, out, dec_ws)
    assert B.tca_ws_status(dec_ws) == B.TCA_OK
    kk, vv = H.f64(cache.k), H.f64(cache.v)
    for b in range(4):
        for h in range(hq):
            rows = cache.unit_rows(b * hkv + h // (hq // hkv))
            w, a, s = S.masked_attention(H.f64(qn)[b, h][None], kk[rows], vv[rows], np.ones((1, len(rows)), dtype=bool), H.scale_of(d))
            H.check(H.f64(out)[b, h][None], w, S.attention_tolerance(w, a, s, d, np.array([len(rows)]), dtype), "decode")


def test_the_binding_refuses_wrong_tensors():
    prm = H.params(2, 4, 2, 64, "bf16")
    cache = H.make_cache(prm, 5, 5, 0, 20, "bf16", 16)
    q, kd, vd = drafts(prm, 4, "bf16", 130)
    par = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    ws, o, n = B.alloc_tree_workspace(prm, 4), torch.zeros_like(q), np.zeros(2, dtype=np.int32)
    good = dict(q=q, kd=kd, vd=vd, par=par, live=None, o=o, ws=ws)
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(kd=kd[:, :1]), dict(vd=vd.transpose(1, 2)), dict(o=o[:1]),
                dict(par=par.long()), dict(live=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(ws=ws.cpu()),
                dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(par=par.cpu())):
        a = {**good, **bad}
        with pytest.raises(ValueError):
            B.tca_attn_tree(prm, a["q"], a["kd"], a["vd"], 4, a["par"], a["live"], cache, a["o"], a["ws"])
    for bad in (dict(q=q.float()), dict(kd=kd.cpu()), dict(vd=vd[:, :, :3]), dict(par=par.long())):
        a = {**good, **bad}
        with pytest.raises(ValueError):
            B.tca_cache_accept(prm, cache, a["kd"], a["vd"], a["q"], 4, a["par"], n)
    with pytest.raises(ValueError):
        B.tca_cache_accept(prm, cache, kd, vd, q, 4, par, np.zeros(3, dtype=np.int32))
    with pytest.raises(ValueError):
        B.tca_cache_accept(prm, cache, kd, vd, q, 4, par, np.zeros(2, dtype=np.int64))
    x = H.randn(1, (2, 10, 64), "bf16")
    st = torch.tensor([0, 5, 10], device="cuda")
    pws = B.alloc_workspace(prm, 10, B.TCA_OP_PACKED)
    qp = H.randn(2, (4, 10, 64), "bf16")
    for a in ((qp, x, x, st.int(), qp.clone(), pws), (qp, x, x.float(), st, qp.clone(), pws), (qp[:, :9], x, x, st, qp.clone(), pws),
              (qp, x, x, st[:2], qp.clone(), pws), (qp, x, x, st.cpu(), qp.clone(), pws), (qp, x, x, st, qp[:, :, ::2], pws),
              (qp, x.transpose(1, 2).contiguous().transpose(1, 2), x, st, qp.clone(), pws)):
        with pytest.raises(ValueError):
            B.tca_attn_packed(prm, a[0], a[1], a[2], 10, a[3], a[4], a[5])
    with pytest.raises(ValueError):
        B.tca_cache_load(prm, x.cpu(), x, 10, np.array([0, 10]), None, cache)
    torch.cuda.synchronize()


def test_the_binding_refuses_a_cache_made_for_something_else():
    prm = H.params(2, 4, 2, 64, "bf16")
    q, kd, vd = drafts(prm, 4, "bf16", 131)
    par, n = torch.zeros(2, 4, dtype=torch.int32, device="cuda"), np.ones(2, dtype=np.int32)
    ws, x = B.alloc_tree_workspace(prm, 4), H.randn(1, (2, 10, 64), "bf16")
    elsewhere = B.Cache(prm, np.full(4, 20), 96, np.full(4, 4), device="cpu", init=False)
    for cache in (H.make_cache(H.params(2, 4, 2, 64, "f32"), 5, 5, 0, 20, "f32", 17),
                  H.make_cache(H.params(2, 4, 2, 128, "bf16"), 5, 5, 0, 20, "bf16", 17), elsewhere):
        was = cache.k.clone()
        with pytest.raises(ValueError, match="cache"):
            B.tca_attn_tree(prm, q, kd, vd, 4, par, None, cache, torch.zeros_like(q), ws)
        with pytest.raises(ValueError, match="cache"):
            B.tca_cache_accept(prm, cache, kd, vd, q, 4, par, n)
        with pytest.raises(ValueError, match="cache"):
            B.tca_cache_load(prm, x, x, 10, np.array([0, 5, 10]), None, cache)
        assert torch.equal(cache.k, was)
    torch.cuda.synchronize()


def test_calls_on_several_streams_at_once():
    """Prompts of one batch while another one drafts and accepts: each with buffers and workspaces of its own."""
    prm, pp = H.params(2, 8, 2, 128, "bf16"), H.params(3, 6, 2, 128, "bf16")
    starts = [0, 700, 701, 1500]
    qp, kp = H.randn(1, (6, 1500, 128), "bf16"), H.randn(2, (2, 1500, 128), "bf16")
    T, parent = 20, np.stack([H.chain(20), H.bush(20, 4)])
    sets, want = [], H.run_packed(pp, qp, kp, kp, starts)
    for i in range(3):
        cache = H.make_cache(prm, [900, 20, 700, 1], [90, 90, 3, 3], 5, 1200, "bf16", 20 + i, extra_cap=40, t_keep=3)
        sets.append((cache, drafts(prm, T, "bf16", 160 + 3 * i), H.clone_cache(prm, cache)))
    n, path = np.array([20, 7], dtype=np.int32), torch.arange(T, dtype=torch.int32, device="cuda").repeat(2, 1)
    trees = []
    for cache, (q, kd, vd), alone in sets:
        trees.append(H.run_tree(prm, q, kd, vd, parent, alone))
        B.tca_cache_accept(prm, alone, kd, vd, q, T, path, n)
        trees.append(H.run_tree(prm, q, kd, vd, parent, alone))
    par = torch.from_numpy(parent).cuda()
    st = torch.tensor(starts, device="cuda")
    pws, po = B.alloc_workspace(pp, 1500, B.TCA_OP_PACKED), torch.empty_like(qp)
    tws = [B.alloc_tree_workspace(prm, T) for _ in sets]
    out = [torch.empty_like(trees[0]) for _ in trees]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    for i, (cache, (q, kd, vd), _) in enumerate(sets):
        with torch.cuda.stream(streams[i]):
            B.tca_attn_tree(prm, q, kd, vd, T, par, None, cache, out[2 * i], tws[i])
            B.tca_cache_accept(prm, cache, kd, vd, q, T, path, n)
            B.tca_attn_tree(prm, q, kd, vd, T, par, None, cache, out[2 * i + 1], tws[i])
        with torch.cuda.stream(streams[3]):
            B.tca_attn_packed(pp, qp, kp, kp, 1500, st, po, pws)
    torch.cuda.synchronize()
    for a, b in zip(out, trees):
        assert torch.equal(a, b)
    for cache, _, alone in sets:
        H.mirror_equals_device(cache)
        assert torch.equal(cache.state, alone.state) and torch.equal(cache.pos, alone.pos) and torch.equal(cache.k, alone.k)
    assert torch.equal(po, want)
