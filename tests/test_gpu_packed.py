"""tca_attn_packed and tca_cache_load against the oracle: sizes, layouts, masked garbage, replays."""
import numpy as np
import pytest
import torch

import serving_harness as H
from oracle import serving_oracle as S
from paper_2512_09238_b200 import binding as B

pytestmark = pytest.mark.gpu

LENS = {
    "one": [1], "empty_between": [0, 1, 0, 5, 0], "tile_edges": [127, 128, 129, 63, 64, 65],
    "ragged": [300, 1, 33, 0, 511], "hundreds": [(7 * i) % 11 for i in range(290)] + [200], "many": [3, 17, 0, 40, 1, 1, 96, 2] * 6,
}


def case(lens, hq, hkv, d, dtype, layout, seed, lead=3, trail=4):
    starts = lead + np.concatenate([[0], np.cumsum(lens)])
    rows = int(starts[-1]) + trail
    mk = lambda i, h: H.packed_buffer(seed + i, h, rows, d, dtype, layout)  # noqa: E731
    return H.params(len(lens), hq, hkv, d, dtype), mk(0, hq), mk(1, hkv), mk(2, hkv), starts


def compare(prm, q, k, v, starts, o, dtype):
    want, a, s = S.packed_attention(H.f64(q), H.f64(k), H.f64(v), starts, H.scale_of(prm.head_dim))
    n = np.full(want.shape[:2], max(1, int(np.max(np.diff(starts)))))
    H.check(H.f64(o), want, S.attention_tolerance(want, a, s, prm.head_dim, n, dtype), "packed")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(LENS))
def test_lengths(name, d, dtype):
    prm, q, k, v, starts = case(LENS[name], 4, 2, d, dtype, "heads", 10)
    compare(prm, q, k, v, starts, H.run_packed(prm, q, k, v, starts), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8])
def test_groups(group, dtype):
    prm, q, k, v, starts = case([70, 5, 260], 2 * group, 2, 128, dtype, "heads", 20)
    compare(prm, q, k, v, starts, H.run_packed(prm, q, k, v, starts), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 3, 7, 8])
def test_groups_of_short_heads(group, dtype):
    """head_dim 64: a longer ring of tiles; several items per CTA."""
    prm, q, k, v, starts = case([700, 129, 1, 0, 400, 64], group * 4, 4, 64, dtype, "tokens", 25)
    compare(prm, q, k, v, starts, H.run_packed(prm, q, k, v, starts), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    """Heads more than 2^31 bytes apart: element offsets need more than 32 bits."""
    L, d, hq, hkv = 300, 64, 4, 2
    far = (1 << 31) // H.DT[dtype].itemsize + 4096

    def spread(seed, heads):
        buf = torch.zeros(far * (heads - 1) + L * d, dtype=H.DT[dtype], device="cuda")
        x = buf.as_strided((heads, L, d), (far, d, 1))
        x.copy_(H.randn(seed, (heads, L, d), dtype))
        return x

    q, k, v, o = spread(1, hq), spread(2, hkv), spread(3, hkv), spread(4, hq)
    o.fill_(float("nan"))
    prm, starts = H.params(2, hq, hkv, d, dtype), [0, 100, L]
    compare(prm, q, k, v, np.array(starts), H.run_packed(prm, q, k, v, starts, out=o), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["tokens", "fused", "odd"])
@pytest.mark.parametrize("d", [64, 128])
def test_layouts(layout, d, dtype):
    prm, q, k, v, starts = case([200, 31, 1], 6, 3, d, dtype, layout, 30)
    o = H.packed_buffer(33, 6, q.shape[1], d, dtype, layout)
    o.fill_(float("nan"))
    o = H.run_packed(prm, q, k, v, starts, out=o)
    compare(prm, q, k, v, starts, o, dtype)
    # the layout does not change a bit of the result
    c = [x.contiguous() for x in (q, k, v)]
    o2 = H.run_packed(prm, *c, starts)
    assert torch.equal(o.nan_to_num(7.0), o2.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_a_query_does_not_see_have_no_influence(bad, dtype):
    """A sequence's result is the same whatever its neighbours hold, and a row's whatever its later rows hold."""
    prm, q, k, v, starts = case([150, 77, 140], 4, 2, 128, dtype, "heads", 40)
    clean = H.f64(H.run_packed(prm, q, k, v, starts))
    cut = int(starts[1]) + 30                               # row 30 of the second sequence and all behind it
    for x in (k, v):
        x[:, cut:] = bad
        x[:, :int(starts[1]) - 1] = bad                      # all of the first sequence but its last row
        x[:, int(starts[0]) - 1] = bad
    got = H.f64(H.run_packed(prm, q, k, v, starts))
    lo = int(starts[1])
    assert np.array_equal(got[:, lo:cut], clean[:, lo:cut])
    # only values, not keys: the rows that do see the bad value show it
    prm, q, k, v, starts = case([150, 77, 140], 4, 2, 128, dtype, "heads", 41)
    clean = H.f64(H.run_packed(prm, q, k, v, starts))
    v[1, cut, 5] = bad
    got = H.f64(H.run_packed(prm, q, k, v, starts))
    same = np.ones_like(got, dtype=bool)
    same[2:, cut:int(starts[2]), 5] = False
    assert np.array_equal(got[same], clean[same], equal_nan=True)
    hit = got[2:, cut:int(starts[2]), 5]
    assert np.isnan(hit).all() if np.isnan(bad) else (hit == bad).all()


def test_large_scores_and_the_lowest_value():
    """Scores of thousands, and keys at the type's lowest finite value, stay finite."""
    prm, q, k, v, starts = case([90, 200], 4, 2, 64, "bf16", "heads", 50)
    q *= 40
    compare(prm, q, k, v, starts, H.run_packed(prm, q, k, v, starts), "bf16")
    k[:, 40:60] = torch.finfo(torch.bfloat16).min
    q[:] = q.abs().clamp(max=1.0)                            # scores of -1e38 or so: weight zero next to any other key
    out = H.f64(H.run_packed(prm, q, k, v, starts))
    assert np.isfinite(out[:, starts[0]:starts[-1]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_runs_and_another_stream_agree_bit_for_bit(dtype):
    prm, q, k, v, starts = case([513, 64, 300], 8, 2, 128, dtype, "heads", 60)
    a = H.run_packed(prm, q, k, v, starts)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = H.run_packed(prm, q, k, v, starts)
    torch.cuda.synchronize()
    assert torch.equal(a.nan_to_num(3.0), b.nan_to_num(3.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 3, 5, 7, 8])
def test_a_row_rounds_the_same_whatever_shares_its_tile(group, dtype):
    """Bit for bit: a sequence's rows while the other sequences' queries, its own later queries, and the calls
    before (whose queries stay in shared memory behind a group's last whole position) hold large ones."""
    lens = [219, 29, 2, 140, 311, 5, 90]
    prm, q, k, v, starts = case(lens, 2 * group, 2, 128, dtype, "heads", 65)
    q *= 3
    first = H.run_packed(prm, q, k, v, starts)
    for i, n in enumerate(lens):
        lo, hi = int(starts[i]), int(starts[i + 1])
        loud = q * 50
        H.run_packed(prm, loud, k, v, starts)
        keep = lo + (n + 1) // 2
        loud[:, lo:keep] = q[:, lo:keep]
        got = H.run_packed(prm, loud, k, v, starts)
        assert torch.equal(got[:, lo:keep], first[:, lo:keep]), i
        loud[:, lo:hi] = q[:, lo:hi]
        got = H.run_packed(prm, loud, k, v, starts)
        assert torch.equal(got[:, lo:hi], first[:, lo:hi]), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_call_replays_with_other_lengths(dtype):
    prm, q, k, v, starts = case([100, 50, 250], 4, 2, 128, dtype, "heads", 70)
    st = torch.tensor(starts, dtype=torch.int64, device="cuda")
    ws = B.alloc_workspace(prm, q.shape[1], B.TCA_OP_PACKED)
    o = torch.full_like(q, float("nan"))
    B.tca_attn_packed(prm, q, k, v, q.shape[1], st, o, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.tca_attn_packed(prm, q, k, v, q.shape[1], st, o, ws)
    for other in ([3, 3, 203, 403], [0, 399, 400, 407], [5, 5, 5, 5], list(starts)):
        o.fill_(float("nan"))
        st.copy_(torch.tensor(other, dtype=torch.int64))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o.nan_to_num(3.0), H.run_packed(prm, q, k, v, other).nan_to_num(3.0))


def test_offsets_outside_the_buffers_are_clamped():
    prm, q, k, v, _ = case([40, 60], 4, 2, 128, "bf16", "heads", 80)
    rows = q.shape[1]
    a = H.run_packed(prm, q, k, v, [-7, 40, rows + 1000])
    b = H.run_packed(prm, q, k, v, [0, 40, rows])
    assert torch.equal(a.nan_to_num(3.0), b.nan_to_num(3.0))
    c = H.run_packed(prm, q, k, v, [50, 20, 10])             # descending: empty sequences
    assert torch.isnan(c).all()


def test_long_rows_sampled():
    """One long prompt: sampled rows against the oracle (a full fp64 pass would take minutes)."""
    L, hq, hkv, d = 20000, 4, 1, 128
    prm = H.params(2, hq, hkv, d, "bf16")
    q, k, v = (H.packed_buffer(90 + i, h, L + 10, d, "bf16", "heads") for i, h in enumerate((hq, hkv, hkv)))
    o = H.f64(H.run_packed(prm, q, k, v, [0, 10, L + 10]))
    kd, vd, qd = H.f64(k), H.f64(v), H.f64(q)
    for i in (0, 1, 127, 128, 4096, 12345, L - 2, L - 1):
        for h in (0, 3):
            vis = np.ones((1, i + 1), dtype=bool)
            want, a, s = S.masked_attention(qd[h, 10 + i][None], kd[0, 10:11 + i], vd[0, 10:11 + i], vis, H.scale_of(d))
            H.check(o[h, 10 + i][None], want, S.attention_tolerance(want, a, s, d, np.array([i + 1]), "bf16"), f"row {i}")


def test_many_sequences_with_long_ones_among_them():
    """More sequences than are searched in sorted order, and more keys than the L2 holds."""
    hq, hkv, d = 8, 4, 128
    lens = [(i * 37) % 60 for i in range(300)]
    lens[0], lens[150], lens[299] = 5000, 9000, 20000
    prm = H.params(len(lens), hq, hkv, d, "bf16")
    starts = np.concatenate([[0], np.cumsum(lens)])
    rows = int(starts[-1])
    q, k, v = (H.packed_buffer(85 + i, h, rows, d, "bf16", "heads") for i, h in enumerate((hq, hkv, hkv)))
    out = H.run_packed(prm, q, k, v, starts)
    assert torch.isfinite(out).all()
    for s in (0, 7, 150, 151, 298, 299):
        n, lo = lens[s], int(starts[s])
        for i in {0, n // 2, n - 1} if n else ():
            for h in (0, 3, 7):
                kk, vv = H.f64(k[h // 2, lo:lo + i + 1]), H.f64(v[h // 2, lo:lo + i + 1])
                want, a, ss = S.masked_attention(H.f64(q[h, lo + i])[None], kk, vv, np.ones((1, i + 1), dtype=bool), H.scale_of(d))
                H.check(H.f64(out[h, lo + i])[None], want, S.attention_tolerance(want, a, ss, d, np.array([i + 1]), "bf16"), f"{s} {i} {h}")


@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_more_keys_than_the_l2_holds(layout):
    """Enough keys that the heads are worked through one after another; several sequences, all heads sampled."""
    hq, hkv, d = 16, 8, 128
    lens = [9000, 0, 301, 1, 16000, 77, 5000]
    prm = H.params(len(lens), hq, hkv, d, "bf16")
    starts = np.concatenate([[0], np.cumsum(lens)])
    rows = int(starts[-1])
    assert rows * hkv * d * 4 > 100e6
    q, k, v = (H.packed_buffer(95 + i, h, rows, d, "bf16", layout) for i, h in enumerate((hq, hkv, hkv)))
    out = H.run_packed(prm, q, k, v, starts)
    assert torch.isfinite(out).all()                          # every row of every head was written
    for s, n in enumerate(lens):
        for i in {0, n // 3, n - 65, n - 1}:
            if not 0 <= i < n:
                continue
            lo = int(starts[s])
            for h in range(hq):
                kk, vv = H.f64(k[h // 2, lo:lo + i + 1]), H.f64(v[h // 2, lo:lo + i + 1])
                want, a, ss = S.masked_attention(H.f64(q[h, lo + i])[None], kk, vv, np.ones((1, i + 1), dtype=bool), H.scale_of(d))
                H.check(H.f64(out[h, lo + i])[None], want, S.attention_tolerance(want, a, ss, d, np.array([i + 1]), "bf16"), f"{s} {i} {h}")


def test_a_set_status_word_stops_the_call():
    prm, q, k, v, starts = case([50, 60], 4, 2, 128, "bf16", "heads", 97)
    ws = B.alloc_workspace(prm, q.shape[1], B.TCA_OP_PACKED)
    ws[:4] = torch.tensor([1, 0, 0, 0], dtype=torch.uint8, device="cuda")
    o = torch.full_like(q, 7.0)
    B.tca_attn_packed(prm, q, k, v, q.shape[1], torch.tensor(starts, device="cuda"), o, ws)
    assert B.tca_ws_status(ws) == B.TCA_ERR_TIMEOUT and (o == 7.0).all()
    ws.zero_()
    compare(prm, q, k, v, starts, H.run_packed(prm, q, k, v, starts, ws=ws), "bf16")


def test_a_workspace_cleared_by_the_kernel_before():
    """The status word counts as it is when the call's turn comes, not as it was while the kernel before still ran."""
    prm, q, k, v, starts = case([50, 60], 4, 2, 128, "bf16", "heads", 98)
    want = H.run_packed(prm, q, k, v, starts)
    cache = H.make_cache(prm, 200, 90, 0, 300, "bf16", 17)
    par = torch.from_numpy(np.tile(H.chain(5), (2, 1))).cuda()
    qd, kd = H.randn(1, (2, 4, 5, 128), "bf16"), H.randn(2, (2, 2, 5, 128), "bf16")
    tree = H.run_tree(prm, qd, kd, kd, par.cpu().numpy(), cache)
    ws, tws = B.alloc_workspace(prm, q.shape[1], B.TCA_OP_PACKED), B.alloc_tree_workspace(prm, 5)
    st, o, ot = torch.tensor(starts, device="cuda"), torch.empty_like(q), torch.empty_like(qd)
    rows = slice(int(starts[0]), int(starts[-1]))
    for size in (256, 1 << 16, 1 << 22, 1 << 26):             # cleared by a kernel that takes longer and longer
        for w, call, out, right in ((ws, lambda w: B.tca_attn_packed(prm, q, k, v, q.shape[1], st, o, w), o, want),
                                    (tws, lambda w: B.tca_attn_tree(prm, qd, kd, kd, 5, par, None, cache, ot, w), ot, tree)):
            big = torch.zeros(max(size, w.numel()), dtype=torch.uint8, device="cuda")
            mine = big[:w.numel()]
            for _ in range(20):
                out.fill_(7.0)
                mine[:4] = torch.tensor([1, 0, 0, 0], dtype=torch.uint8, device="cuda")
                big.zero_()
                call(mine)
                assert B.tca_ws_status(mine) == B.TCA_OK
                cut = (slice(None), rows) if out is o else slice(None)
                assert torch.equal(out[cut], right[cut])


def test_tensor_cores_agree_with_the_fp32_pipes():
    prm, q, k, v, starts = case([700, 130, 9], 8, 2, 128, "bf16", "tokens", 100)
    a = H.f64(H.run_packed(prm, q, k, v, starts))
    prm2 = H.params(3, 8, 2, 128, "bf16", flags=B.TCA_FLAG_PREFILL_SIMT)
    b = H.f64(H.run_packed(prm2, q, k, v, starts))
    want, aa, s = S.packed_attention(H.f64(q), H.f64(k), H.f64(v), starts, H.scale_of(128))
    tol = 2 * S.attention_tolerance(want, aa, s, 128, np.full(want.shape[:2], 700), "bf16")
    H.check(a, b, tol, "tensor cores against FP32 pipes")


# ------------------------------------------------------------------ tca_cache_load
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["heads", "tokens", "fused", "odd"])
def test_load_places_every_row(layout, d, dtype):
    lens, slots, hkv = [100, 0, 97, 1, 400], np.array([4, 0, 2, 6, 5], dtype=np.int32), 3
    prm = H.params(7, 2 * hkv, hkv, d, dtype, block=32, window=64)
    starts = 2 + np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    k, v = (H.packed_buffer(i, hkv, int(starts[-1]) + 3, d, dtype, layout) for i in (1, 2))
    cache = H.make_cache(prm, 10, 50, 7, 60, dtype, 5, extra_cap=400)
    before = H.clone_cache(prm, cache)
    B.tca_cache_load(prm, k, v, k.shape[1], starts, slots, cache)
    torch.cuda.synchronize()
    H.mirror_equals_device(cache)
    want = {n: getattr(before, n).clone() for n in ("k", "v", "pos")}
    for i, n in enumerate(lens):
        g, t = S.load_split(n, prm.window, prm.block)
        for h in range(hkv):
            u = int(slots[i]) * hkv + h
            assert (cache.n_global[u], cache.n_tail[u], cache.tail_head[u], cache.seq_len[u]) == (g, t, 0, n)
            rows = torch.from_numpy(cache.unit_rows(u)).cuda()
            src = slice(int(starts[i]), int(starts[i]) + n)
            want["k"][rows], want["v"][rows] = k[h, src], v[h, src]
            want["pos"][rows] = torch.arange(n, dtype=torch.int32, device="cuda")
    for n in ("k", "v", "pos"):
        assert torch.equal(getattr(cache, n), want[n]), n    # sequences 1 and 3 and all unused rows as they were


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_load_equals_compaction_of_everything(dtype):
    L, hkv, d, batch = 333, 2, 128, 2
    prm = H.params(batch, 4, hkv, d, dtype, block=32, window=64)
    k, v = (H.randn(i, (batch, hkv, L, d), dtype) for i in (1, 2))
    g, t = S.load_split(L, 64, 32)
    cap = np.full(batch * hkv, g, dtype=np.int64)
    a, b = (B.Cache(prm, cap, 96, np.full(batch * hkv, 4, dtype=np.int64)) for _ in range(2))
    offs = np.arange(batch * hkv + 1, dtype=np.int64) * g
    idx = torch.arange(g, dtype=torch.int32, device="cuda").repeat(batch * hkv)
    B.tca_compact_kv(prm, k, v, L, idx, torch.from_numpy(offs).cuda(), offs, a)
    pk, pv = (x.transpose(0, 1).reshape(hkv, batch * L, d).contiguous() for x in (k, v))
    B.tca_cache_load(prm, pk, pv, batch * L, np.arange(batch + 1, dtype=np.int64) * L, None, b)
    torch.cuda.synchronize()
    for n in ("k", "v", "pos", "state"):
        assert torch.equal(getattr(a, n), getattr(b, n)), n
    H.mirror_equals_device(b)


def test_load_of_more_sequences_than_one_launch_takes():
    batch, d = 250, 64
    prm = H.params(batch, 1, 1, d, "bf16", block=16, window=8)
    lens = np.arange(batch) % 37
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    k, v = (H.randn(i, (1, int(starts[-1]), d), "bf16") for i in (1, 2))
    cache = B.Cache(prm, np.full(batch, 32, dtype=np.int64), 24, np.ones(batch, dtype=np.int64))
    slots = np.random.default_rng(0).permutation(batch).astype(np.int32)
    B.tca_cache_load(prm, k, v, int(starts[-1]), starts, slots, cache)
    torch.cuda.synchronize()
    H.mirror_equals_device(cache)
    for i in range(batch):
        rows = torch.from_numpy(cache.unit_rows(int(slots[i]))).cuda()
        assert torch.equal(cache.k[rows], k[0, starts[i]:starts[i + 1]]) and torch.equal(cache.v[rows], v[0, starts[i]:starts[i + 1]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_load_far_into_a_large_cache(dtype):
    """The second sequence's rows lie more than 2^31 elements behind the first's."""
    d, far = 128, (1 << 31) // 128 // 2 + 1000
    prm = H.params(2, 2, 2, d, dtype, block=32, window=64)
    cache = B.Cache(prm, np.array([far, far, 512, 512]), 96, np.full(4, 4))
    assert int(cache.seg_start[2]) * d > 1 << 31
    k, v = (H.randn(i, (2, 500, d), dtype) for i in (1, 2))
    B.tca_cache_load(prm, k, v, 500, np.array([20, 500], dtype=np.int64), np.array([1], dtype=np.int32), cache)
    torch.cuda.synchronize()
    H.mirror_equals_device(cache)
    for h in range(2):
        rows = torch.from_numpy(cache.unit_rows(2 + h)).cuda()
        assert torch.equal(cache.k[rows], k[h, 20:]) and torch.equal(cache.v[rows], v[h, 20:])
        assert torch.equal(cache.pos[rows], torch.arange(480, dtype=torch.int32, device="cuda"))
    assert not cache.k[:1000].any() and not cache.k[-1].any()


def test_load_refuses_without_touching_anything():
    prm = H.params(3, 2, 1, 64, "bf16", block=32, window=64)
    k = H.randn(1, (1, 500, 64), "bf16")
    cache = H.make_cache(prm, 10, 5, 0, 15, "bf16", 5, extra_cap=90)
    before = H.clone_cache(prm, cache)
    i64, i32 = (lambda *x: np.array(x, dtype=np.int64)), (lambda *x: np.array(x, dtype=np.int32))
    for starts, slots, status in (
            (i64(0, 10, 20), i32(1, 1), B.TCA_ERR_INVALID_ARG), (i64(0, 10, 20), i32(0, 3), B.TCA_ERR_INVALID_ARG),
            (i64(0, 10, 501), i32(0, 1), B.TCA_ERR_INVALID_ARG), (i64(10, 5), None, B.TCA_ERR_INVALID_ARG),
            (i64(-1, 5), None, B.TCA_ERR_INVALID_ARG), (i64(0, 1, 2, 3, 4), None, B.TCA_ERR_INVALID_ARG),
            (i64(0, 10, 210), i32(0, 1), B.TCA_ERR_CAPACITY)):
        with pytest.raises(B.TcaError) as e:
            B.tca_cache_load(prm, k, k, 500, starts, slots, cache)
        assert e.value.status == status
    torch.cuda.synchronize()
    for n in ("k", "v", "pos", "state"):
        assert torch.equal(getattr(cache, n), getattr(before, n))
    H.mirror_equals_device(cache)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_batch_without_a_token(dtype):
    prm = H.params(3, 4, 2, 64, dtype)
    cache = H.make_cache(prm, 10, 20, 3, 30, dtype, 95)
    q, k = H.randn(1, (4, 0, 64), dtype), H.randn(2, (2, 0, 64), dtype)
    assert H.run_packed(prm, q, k, k, [0, 0, 0, 0]).numel() == 0
    before = cache.state.clone()
    B.tca_cache_load(prm, k, k, 0, np.zeros(2, dtype=np.int64), np.array([1], dtype=np.int32), cache)
    after = cache.state.view(6, -1).cpu().numpy()
    assert list(cache.n_tail) == [20, 20, 0, 0, 20, 20] and list(cache.n_global) == [10, 10, 0, 0, 10, 10]
    assert np.array_equal(after[[0, 1, 4, 5]], before.view(6, -1).cpu().numpy()[[0, 1, 4, 5]])
    H.mirror_equals_device(cache)


# ------------------------------------------------------------------ decode over a place that was used before
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_decode_after_a_place_is_reused(bad, d, dtype):
    """A prompt that takes the place of one that held infinities or NaN decodes as in a cache that is new."""
    hq, hkv = 8, 2
    prm = H.params(3, hq, hkv, d, dtype, block=32, window=64)
    cap, keep = np.full(6, 512, dtype=np.int64), np.full(6, 4, dtype=np.int64)
    long = H.randn(1, (hkv, 600, d), dtype)
    long[:] = bad
    q, other = H.randn(2, (3, hq, d), dtype, 1.5), H.randn(3, (hkv, 150, d), dtype)
    load = lambda c, x, n, slot: B.tca_cache_load(prm, x, x, x.shape[1], np.array([0, n], dtype=np.int64), np.array([slot], dtype=np.int32), c)  # noqa: E731
    for n in (1, 15, 17, 100, 129, 417):
        x = H.randn(10 + n, (hkv, n, d), dtype)
        out = []
        for used in (True, False):
            cache = B.Cache(prm, cap, 96, keep)
            if used:
                load(cache, long, 600, 1)
            load(cache, other, 150, 0)
            load(cache, other, 150, 2)
            load(cache, x, n, 1)
            o, ws = torch.full_like(q, float("nan")), B.alloc_workspace(prm, cache.rows_total, B.TCA_OP_DECODE)
            B.tca_attn_decode(prm, q, cache, o, ws)
            assert B.tca_ws_status(ws) == B.TCA_OK
            out.append(o)
        assert torch.isfinite(out[0]).all() and torch.equal(out[0], out[1]), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 4, 8])
def test_decode_rows_not_in_use_have_no_influence(group, dtype):
    """Everything behind the ends of the runs, wrapped rings among them, may hold anything; with and without a workspace."""
    prm = H.params(2, 3 * group, 3, 128, dtype)
    cache = H.make_cache(prm, [70, 300, 129, 1, 0, 1000], [90, 30, 96, 20, 95, 11], [50, 0, 20, 90, 3, 94], 1500, dtype, 8, extra_cap=40, tail_cap=97)
    q, ws = H.randn(7, (2, 3 * group, 128), dtype, 1.5), B.alloc_workspace(prm, cache.rows_total, B.TCA_OP_DECODE)

    def both():
        a, b = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
        B.tca_attn_decode(prm, q, cache, a, ws)
        B.tca_attn_decode_static(prm, q, cache, b)
        assert B.tca_ws_status(ws) == B.tca_decode_static_status() == B.TCA_OK
        return a, b

    clean = both()
    unused = torch.ones(cache.rows_total, dtype=torch.bool, device="cuda")
    for u in range(6):
        unused[torch.from_numpy(cache.unit_rows(u)).cuda()] = False
    for bad in (float("nan"), float("inf"), -float("inf")):
        cache.k[unused], cache.v[unused] = bad, bad
        for got, want in zip(both(), clean):
            assert torch.isfinite(got).all() and torch.equal(got, want)
    # nor does the other sequence, whose rows begin where the first one's ring ends
    theirs = torch.zeros(cache.rows_total, dtype=torch.bool, device="cuda")
    theirs[int(cache.seg_start[3]):] = True
    keep = [x[theirs].clone() for x in (cache.k, cache.v)]
    cache.k[theirs], cache.v[theirs] = float("nan"), float("inf")
    for got, want in zip(both(), clean):
        assert torch.equal(got[0], want[0])
    cache.k[theirs], cache.v[theirs] = keep
    # the last row in use does show
    cache.v[int(cache.unit_rows(1)[-1]), 5] = float("inf")
    assert torch.isinf(both()[0][0, group:2 * group, 5]).all()


# ------------------------------------------------------------------ a prompt alone and in a batch
@pytest.mark.parametrize("dtype,flags", [("f32", 0), ("bf16", 0), ("bf16", B.TCA_FLAG_PREFILL_SIMT)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 4])
def test_a_prompt_rounds_the_same_alone_and_in_any_batch(group, d, dtype, flags):
    """Bit for bit, while the batch and the buffers around it go from a few rows to thousands (other tile shapes,
    another order of the heads) and to more sequences than are searched in sorted order."""
    hkv = 2
    hq = hkv * group
    rows = 24000 // hq + 800
    q, k, v = (H.randn(i, (h, rows, d), dtype, 1.5) for i, h in ((1, hq), (2, hkv), (3, hkv)))
    for n in (1, 40, 64, 65, 100, 129, 200, 333, 700):
        def run(at, starts, total):
            """The prompt at row `at` of buffers of `total` rows, among the given sequences."""
            a, b, c = (torch.cat([x[:, 700:700 + at], x[:, :n], x[:, 700 + at:700 + total - n]], dim=1) for x in (q, k, v))
            o = H.run_packed(H.params(len(starts) - 1, hq, hkv, d, dtype, flags=flags), a, b, c, starts)
            return o[:, at:at + n]
        alone = run(0, [0, n], n)
        assert torch.isfinite(alone).all()
        full = rows - 700 + n
        assert torch.equal(run(0, [0, n], full), alone), (n, "much padding")
        assert torch.equal(run(500, [0, 500, 500 + n, full], full), alone), (n, "between long prompts")
        many = np.concatenate([np.arange(0, 300, 2), [300, 300 + n, full]])
        assert torch.equal(run(300, many, full), alone), (n, "among many")
