"""The paged cache on the GPU: tca_paged_append, tca_attn_paged and tca_paged_evict against the oracle, alone and together."""
import numpy as np
import pytest
import torch

import paged_harness as Q
import serving_harness as H
from oracle import paged_oracle as P
from paper_2512_09238_b200 import binding as B

pytestmark = pytest.mark.gpu
DTYPES = ["bf16", "f32"]


# ------------------------------------------------------------------ attention
LENS = {"one": [1, 1, 1, 1], "empty": [0, 0, 0, 0], "edges": [15, 16, 17, 127, 128, 129, 255, 256, 257, 0, 63, 1],
        "ragged": [700, 3, 0, 1500, 90, 16], "long": [9000, 1, 5000, 0]}


def query(prm, seed, dtype):
    return H.randn(seed, (prm.batch, prm.n_q_heads, prm.head_dim), dtype, 1.5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("name", list(LENS))
def test_lengths_and_pages(name, page, dtype):
    lens = LENS[name]
    prm = Q.params(len(lens) // 2, 4, 2, 128 if page > 32 else 64, dtype)
    c = Q.make(prm, lens, page, dtype, 5, garbage=float("nan"))
    before = Q.snapshot(c)
    q = query(prm, 1, dtype)
    o = Q.attend(prm, q, c, accumulate=True)
    Q.check(prm, q, c, o, 0, dtype, before)
    again = Q.attend(prm, q, c)
    assert torch.equal(o, again)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8])
def test_groups(group, d, dtype):
    prm = Q.params(2, 3 * group, 3, d, dtype)
    c = Q.make(prm, [300, 40, 1, 0, 129, 1000], 32, dtype, 7)
    before, q = Q.snapshot(c), query(prm, 2, dtype)
    Q.check(prm, q, c, Q.attend(prm, q, c, accumulate=True), 0, dtype, before)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (5, 3), (16, 0), (100, 4), (128, 128), (129, 200), (300, 130), (1000, 1), (7, 4000),
                                           (1, (1 << 31) - 1)])
@pytest.mark.parametrize("page", [16, 128])
def test_windows_and_sinks(page, window, n_sink, dtype):
    prm = Q.params(2, 4, 2, 64, dtype, window)
    c = Q.make(prm, [1, 400, 133, 2000], page, dtype, 9)
    # what the window hides may hold anything, and its pages need not exist
    s = Q.lens_of(c)
    hide = []
    for u in range(4):
        hidden = np.setdiff1d(np.arange(s[u]), P.visible_slots(int(s[u]), window, n_sink))
        hide.append(Q.pool_rows(c, u, hidden))
        gone = [p for p in range(-(-int(s[u]) // page)) if np.isin(np.arange(p * page, min((p + 1) * page, s[u])), hidden).all()]
        c.table[u, gone] = -1 if u % 2 else 1 << 30
    rows = torch.from_numpy(np.concatenate(hide)).cuda()
    c.k.view(-1, 64)[rows], c.v.view(-1, 64)[rows] = float("inf"), float("nan")
    before, q = Q.snapshot(c), query(prm, 3, dtype)
    o = Q.attend(prm, q, c, n_sink, accumulate=True)
    Q.check(prm, q, c, o, n_sink, dtype, before)


@pytest.mark.parametrize("dtype", DTYPES)
def test_bad_pages_are_reported_and_count_as_hidden(dtype):
    prm = Q.params(2, 2, 1, 128, dtype)
    c = Q.make(prm, [500, 300], 32, dtype, 11)
    q = query(prm, 4, dtype)
    c.table[0, 3], c.table[0, 15], c.table[1, 0] = c.n_pages, -5, (1 << 31) - 1
    hidden = [np.concatenate([np.arange(96, 128), np.arange(480, 512)]), np.arange(32)]
    before = Q.snapshot(c)
    o = Q.attend(prm, q, c, accumulate=True, status=B.TCA_ERR_BOUNDS)
    Q.check(prm, q, c, o, 0, dtype, before, hidden)


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_and_nans_in_visible_rows(dtype):
    """-inf scores weigh nothing, a NaN or +inf score makes its heads NaN, an infinite value reaches the result."""
    prm = Q.params(4, 1, 1, 64, dtype)
    c = Q.make(prm, [200] * 4, 16, dtype, 13)
    q = torch.ones(4, 1, 64, dtype=H.DT[dtype], device="cuda")
    k, v = c.k.view(-1, 64), c.v.view(-1, 64)
    r = [torch.from_numpy(Q.pool_rows(c, u, np.arange(200))).cuda() for u in range(4)]
    k[r[0][50]] = float("-inf")
    k[r[1][50]] = float("nan")
    k[r[2][150], 3] = float("inf")
    v[r[3][10], 5] = float("inf")
    o = Q.attend(prm, q, c, accumulate=True).float().cpu()
    assert torch.isfinite(o[0]).all() and torch.isnan(o[1]).all() and torch.isnan(o[2]).all()
    assert o[3, 0, 5] == float("inf") and torch.isfinite(o[3, 0, :5]).all()
    mass = c.mass.view(-1)
    assert torch.isnan(mass[r[1]]).all() and torch.isfinite(mass[r[0]]).all()
    # a unit all of whose scores are -inf has no weights: NaN, not zero
    k[r[0]] = float("-inf")
    assert torch.isnan(Q.attend(prm, q, c)[0].float()).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_offsets_past_32_bits(dtype):
    """A pool of more than 2^31 bytes a buffer (and 2^31 elements in bf16): pages at its far end."""
    prm = Q.params(1, 4, 1, 128, dtype)
    page = 256
    n_pages = (1 << 31) // (page * 128) + 300 if dtype == "bf16" else (1 << 31) // (page * 512) + 300
    c = B.PagedCache(prm, n_pages, page, 4)
    c.free = list(range(n_pages))                    # dealt from the end
    c.reserve([700])
    rows = torch.from_numpy(Q.pool_rows(c, 0, np.arange(700))).cuda()
    c.k.view(-1, 128)[rows], c.v.view(-1, 128)[rows] = H.randn(1, (700, 128), dtype), H.randn(2, (700, 128), dtype)
    c.state[0, 0] = 700
    q = query(prm, 5, dtype)
    o = Q.attend(prm, q, c, accumulate=True)
    k, v = H.f64(c.k.view(-1, 128)[rows]), H.f64(c.v.view(-1, 128)[rows])
    want, a, s, w = P.paged_attention(H.f64(q)[0], k, v, H.scale_of(128))
    H.check(H.f64(o)[0], want, P.paged_tolerance(want, a, s, 128, 700, dtype), "far pages")
    H.check(H.f64(c.mass.view(-1)[rows]), w, P.mass_tolerance(np.zeros(700), w, s, 128, 700), "mass")


@pytest.mark.parametrize("units", [300, 1500])
def test_many_units(units):
    """More units than threads and than pieces of a round; most of them short or empty."""
    prm = Q.params(units, 1, 1, 64, "bf16")
    r = np.random.default_rng(units)
    lens = np.where(r.random(units) < 0.4, 0, r.integers(1, 40, units))
    lens[units // 2] = 5000 if units > 1000 else 300
    c = Q.make(prm, lens, 16, "bf16", 15)
    before, q = Q.snapshot(c), query(prm, 6, "bf16")
    Q.check(prm, q, c, Q.attend(prm, q, c, accumulate=True), 0, "bf16", before)


def test_more_pieces_than_a_round_holds():
    """One share of very many one-step units (64 pieces a round)."""
    n = 148 * 70 + 13
    prm = Q.params(n, 1, 1, 64, "bf16")
    c = Q.make(prm, np.full(n, 3), 16, "bf16", 16)
    before, q = Q.snapshot(c), query(prm, 7, "bf16")
    Q.check(prm, q, c, Q.attend(prm, q, c, accumulate=True), 0, "bf16", before)


@pytest.mark.parametrize("n,filled", [(148 * 140 + 5, 1.0), (50000, 0.3)])
def test_units_by_the_ten_thousand(n, filled):
    """Several rounds of pieces; more units than a share holds the lengths of, and than all threads together."""
    prm = Q.params(n, 1, 1, 64, "bf16")
    r = np.random.default_rng(n)
    c = Q.make(prm, np.where(r.random(n) < filled, r.integers(1, 16, n), 0), 16, "bf16", 17)
    before, q = Q.snapshot(c), query(prm, 8, "bf16")
    Q.check(prm, q, c, Q.attend(prm, q, c), 0, "bf16")
    Q.check(prm, q, c, Q.attend(prm, q, c, accumulate=True), 0, "bf16", before)


@pytest.mark.parametrize("dtype", DTYPES)
def test_long_and_short_pieces_in_a_share(dtype):
    """Shares of 25 steps and more: pieces longer than the ring of stages, short ones in between."""
    prm = Q.params(7, 2, 1, 64, dtype)
    c = Q.make(prm, [200000, 300, 130000, 40, 1, 140000, 900], 128, dtype, 19)
    before, q = Q.snapshot(c), query(prm, 10, dtype)
    Q.check(prm, q, c, Q.attend(prm, q, c, accumulate=True), 0, dtype, before)


@pytest.mark.parametrize("dtype", DTYPES)
def test_shared_pages(dtype):
    """Two sequences read the same pages of a common beginning."""
    prm = Q.params(2, 4, 1, 64, dtype)
    c = Q.make(prm, [200, 330], 32, dtype, 17)
    c.table_host[1, :4] = c.table_host[0, :4]
    c.table.copy_(torch.from_numpy(c.table_host))
    q = query(prm, 8, dtype)
    Q.check(prm, q, c, Q.attend(prm, q, c), 0, dtype)


def test_a_status_word_that_stops_the_call_leaves_results_alone():
    prm = Q.params(2, 8, 2, 128, "bf16")
    c = Q.make(prm, [900, 20, 0, 4000], 64, "bf16", 21)
    ws, q = B.alloc_paged_workspace(prm, c, True), query(prm, 11, "bf16")
    good, before = Q.attend(prm, q, c, ws=ws), Q.snapshot(c)
    ws[0] = 1
    o = torch.full_like(q, 7.0)
    B.tca_attn_paged(prm, q, c, 0, True, o, ws)
    assert B.tca_ws_status(ws) == B.TCA_ERR_TIMEOUT and (o == 7).all()
    Q.same(before, Q.snapshot(c))
    ws.zero_()
    assert torch.equal(good, Q.attend(prm, q, c, ws=ws))


def test_calls_on_several_streams_at_once():
    """Caches, workspaces and tensors of their own."""
    work = []
    for i in range(4):
        prm = Q.params(2, 8, 2, 128, "bf16")
        c = Q.make(prm, [700 + 300 * i, 20, 5000, 64], 32, "bf16", 80 + i)
        q = query(prm, 90 + i, "bf16")
        work.append((prm, c, q, torch.full_like(q, float("nan")), B.alloc_paged_workspace(prm, c), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for prm, c, q, o, ws, stream in work:
            with torch.cuda.stream(stream):
                B.tca_attn_paged(prm, q, c, 0, False, o, ws)
    torch.cuda.synchronize()
    for prm, c, q, o, ws, _ in work:
        assert B.tca_ws_status(ws) == B.TCA_OK
        Q.check(prm, q, c, o, 0, "bf16")


def test_one_workspace_for_calls_of_both_kinds_and_another_stream():
    prm = Q.params(3, 8, 2, 128, "bf16")
    c = Q.make(prm, [900, 20, 0, 400, 3000, 77], 64, "bf16", 18)
    ws, q = B.alloc_paged_workspace(prm, c, True), query(prm, 9, "bf16")
    first = Q.attend(prm, q, c, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = Q.attend(prm, q, c, accumulate=True, ws=ws)
    side.synchronize()
    assert torch.equal(first, second) and torch.equal(first, Q.attend(prm, q, c, ws=ws))


def test_one_workspace_for_caches_of_different_sizes():
    """Many units beside few, so that whatever the layout depends on lies elsewhere."""
    calls = []
    for i, (batch, hq, hkv, d, dtype, lens) in enumerate([(3, 8, 2, 128, "bf16", [9000, 20, 0, 400, 3000, 77]),
                                                          (150, 16, 4, 128, "bf16", [1 + 13 * u % 900 for u in range(600)]),
                                                          (2, 2, 2, 64, "f32", [2000, 5, 130, 700])]):
        prm = Q.params(batch, hq, hkv, d, dtype)
        calls.append((prm, Q.make(prm, lens, 32, dtype, 100 + i), query(prm, 110 + i, dtype), dtype))
    n = max(B.tca_attn_paged_workspace_bytes(prm, c, True) for prm, c, _, _ in calls)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    for accumulate in (False, True, False):
        for prm, c, q, dtype in calls + calls[::-1]:
            before = Q.snapshot(c)
            Q.check(prm, q, c, Q.attend(prm, q, c, accumulate=accumulate, ws=ws), 0, dtype, before if accumulate else None)


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["heads", "tokens", "fused", "odd"])
@pytest.mark.parametrize("page", [16, 256])
def test_append_prompts(page, layout, dtype):
    d, hkv = (64, 3) if dtype == "f32" else (128, 2)
    prm = Q.params(5, hkv, hkv, d, dtype)
    new, slots, held = [300, 0, 1, 129], [4, 1, 0, 2], [7, 100, 0, 33, 255]
    c = Q.make(prm, np.repeat(held, hkv), page, dtype, 20, room=310, seen=np.repeat(held, hkv) * 2)
    starts = np.array(2 + np.concatenate([[0], np.cumsum(new)]), dtype=np.int64)
    rows = int(starts[-1]) + 3
    k, v = (H.packed_buffer(21 + i, hkv, rows, d, dtype, layout) for i in range(2))
    mass = torch.rand(hkv, rows, device="cuda") if layout != "heads" else None
    before = Q.snapshot(c)
    B.tca_paged_append(prm, k, v, rows, starts, np.array(slots, dtype=np.int32), mass, c)
    assert B.tca_paged_status(c)[0] == B.TCA_OK
    want = before
    for i, (n, s) in enumerate(zip(new, slots)):
        for h in range(hkv):
            u = s * hkv + h
            r = Q.pool_rows(c, u, held[s] + np.arange(n))
            lo = int(starts[i])
            want["k"][r], want["v"][r] = H.f64(k[h, lo:lo + n]), H.f64(v[h, lo:lo + n])
            want["pos"][r] = 2 * held[s] + np.arange(n)
            want["mass"][r] = 0 if mass is None else mass[h, lo:lo + n].cpu().numpy()
            want["state"][u, :2] += n
    Q.same(want, Q.snapshot(c))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("placed", [False, True])
def test_append_one_row_each(placed, d, dtype):
    hkv, n = 3, 70
    prm = Q.params(n, hkv, hkv, d, dtype)
    held = np.arange(n) % 40
    c = Q.make(prm, np.repeat(held, hkv), 16, dtype, 24, room=1)
    take = 50 if placed else n
    slots = np.random.default_rng(1).permutation(n)[:take].astype(np.int32) if placed else None
    k, v = H.packed_buffer(25, hkv, take, d, dtype, "tokens"), H.packed_buffer(26, hkv, take, d, dtype, "fused")
    want = Q.snapshot(c)
    B.tca_paged_append(prm, k, v, take, None, slots, None, c)
    for i in range(take):
        s = int(slots[i]) if placed else i
        for h in range(hkv):
            r = Q.pool_rows(c, s * hkv + h, [held[s]])
            want["k"][r], want["v"][r], want["pos"][r], want["mass"][r] = H.f64(k[h, i]), H.f64(v[h, i]), held[s], 0
            want["state"][s * hkv + h, :2] += 1
    Q.same(want, Q.snapshot(c))


def test_append_many_sequences_in_several_launches():
    prm = Q.params(700, 1, 1, 64, "f32")
    for one in (True, False):
        c = Q.make(prm, np.zeros(700, dtype=np.int64), 16, "f32", 27, room=3)
        new = [1] * 600 if one else [i % 4 for i in range(600)]
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        slots = np.random.default_rng(2).permutation(700)[:600].astype(np.int32)
        rows = int(starts[-1])
        k, v = H.randn(28, (1, rows, 64), "f32"), H.randn(29, (1, rows, 64), "f32")
        B.tca_paged_append(prm, k, v, rows, None if one else starts, slots, None, c)
        s = Q.snapshot(c)
        for i in range(600):
            r = Q.pool_rows(c, int(slots[i]), np.arange(new[i]))
            np.testing.assert_array_equal(s["k"][r], H.f64(k[0, starts[i]:starts[i + 1]]))
            np.testing.assert_array_equal(s["v"][r], H.f64(v[0, starts[i]:starts[i + 1]]))
            assert s["state"][slots[i], 0] == new[i]


@pytest.mark.parametrize("one", [True, False])
def test_append_without_room_or_page(one):
    n = 1 if one else 200
    prm = Q.params(4, 1, 1, 64, "bf16")
    c = Q.make(prm, [256 - n + 1, 256 - n, 40, 10], 16, "bf16", 30, room=0, spare=64, max_pages=16)
    c.reserve([256, 256, 256 if not one else 48, 256])
    before = Q.snapshot(c)
    if one:
        c.table[2, 2] = c.n_pages
    else:
        c.table[2, 9] = -1
    k, v = H.randn(31, (1, 4 * n, 64), "bf16"), H.randn(32, (1, 4 * n, 64), "bf16")
    starts = None if one else np.arange(5, dtype=np.int64) * n
    B.tca_paged_append(prm, k, v, 4 * n, starts, None, None, c)
    st, detail = B.tca_paged_status(c)
    assert st == B.TCA_ERR_BOUNDS and detail.tolist() == [0, 1]
    s = Q.snapshot(c)
    np.testing.assert_array_equal(s["state"][:, :2], before["state"][:, :2] + np.array([[0], [n], [0], [n]]))
    assert s["state"][:, 2].tolist() == [1, 0, 2, 0] and s["state"][:, 3].tolist() == [0, 0, 0, 0]
    for u in range(4):       # what was in use is as it was
        r = Q.pool_rows(c, u, np.arange(before["state"][u, 0]))
        for name in ("k", "v", "pos", "mass"):
            np.testing.assert_array_equal(s[name][r], before[name][r])
    c.state[:, 2] = 0
    if not one:              # the page is there now: the same rows go in
        c.table.copy_(torch.from_numpy(c.table_host))
        B.tca_paged_append(prm, k, v, 4 * n, np.array([0, 0, 0, n, n], dtype=np.int64), None, None, c)
        assert B.tca_paged_status(c)[0] == B.TCA_OK and c.state[2, 0].item() == 40 + n


# ------------------------------------------------------------------ evict
def evict_and_check(prm, c, n_sink, n_recent, budgets, refused=()):
    before, lens = Q.snapshot(c), Q.lens_of(c)
    B.tca_paged_evict(prm, c, n_sink, n_recent, torch.tensor(np.asarray(budgets), dtype=torch.int32, device="cuda"))
    st, detail = B.tca_paged_status(c)
    assert st == (B.TCA_ERR_BOUNDS if refused else B.TCA_OK)
    want = {k: x.copy() for k, x in before.items()}
    for u, n in enumerate(lens):
        src = P.evict(before["mass"][Q.pool_rows(c, u, np.arange(n))], before["pos"][Q.pool_rows(c, u, np.arange(n))], int(budgets[u]), n_sink, n_recent)
        if u in refused:
            assert src is None
            want["state"][u, 2] = 3
            continue
        to, frm = Q.pool_rows(c, u, np.arange(len(src))), Q.pool_rows(c, u, src)
        for name in ("k", "v", "pos", "mass"):
            want[name][to] = before[name][frm]
        want["state"][u, 0] = len(src)
    Q.same(want, Q.snapshot(c))


def scramble(c, seed, ties=False):
    """Positions in no order (as earlier evictions leave them), weights with many equal ones."""
    r = np.random.default_rng(seed)
    pos, mass = c.pos.cpu().numpy().reshape(-1), c.mass.cpu().numpy().reshape(-1)
    for u, n in enumerate(Q.lens_of(c)):
        rows = Q.pool_rows(c, u, np.arange(n))
        pos[rows] = r.permutation(3 * int(n))[:n]
        mass[rows] = r.integers(0, 3, n) if ties else np.exp(2 * r.normal(size=n))
    c.pos.copy_(torch.from_numpy(pos).view(c.pos.shape))
    c.mass.copy_(torch.from_numpy(mass).view(c.mass.shape))


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_evict(page, dtype, ties):
    prm = Q.params(3, 4, 4, 64 if dtype == "f32" else 128, dtype)
    lens = [1, 2, 33, 100, 513, 600, 1000, 1025, 2049, 3000, 0, 64]
    c = Q.make(prm, lens, page, dtype, 40)
    scramble(c, 41, ties)
    budgets = [1, 1, 32, 100, 40, 599, 500, 1, 2000, 700, 5, 0]
    evict_and_check(prm, c, 0, 0, budgets)


@pytest.mark.parametrize("n_sink,n_recent", [(0, 1), (4, 0), (4, 50), (300, 10), (1, 5000), (2000, 0)])
def test_evict_keeps_sinks_and_recent_rows(n_sink, n_recent):
    prm = Q.params(1, 4, 4, 64, "bf16")
    c = Q.make(prm, [700, 1500, 900, 1400], 32, "bf16", 42)
    scramble(c, 43)
    lens = Q.lens_of(c)
    pos = c.pos.cpu().numpy().reshape(-1)
    safe = [int(np.sum((np.arange(n) < n_sink) | (pos[Q.pool_rows(c, u, np.arange(n))] > pos[Q.pool_rows(c, u, np.arange(n))].max() - n_recent)))
            for u, n in enumerate(lens)]
    budgets = [safe[0], safe[1] + 1 if safe[1] < lens[1] else lens[1], max(0, safe[2] - 1), min(lens[3], safe[3] + 200)]
    refused = [2] if safe[2] > 0 and budgets[2] < lens[2] else []
    evict_and_check(prm, c, n_sink, n_recent, budgets, refused)


def test_evict_orders_nan_zero_and_signs():
    prm = Q.params(1, 1, 1, 64, "f32")
    c = Q.make(prm, [12], 16, "f32", 44)
    w = [0.0, -0.0, float("nan"), 1.0, float("inf"), -1.0, 0.0, -0.0, float("-inf"), 1e-45, -float("nan"), 1.0]
    for budget in range(12):
        c.state[0, 0] = 12
        c.mass.view(-1)[torch.from_numpy(Q.pool_rows(c, 0, np.arange(12))).cuda()] = torch.tensor(w, device="cuda")
        evict_and_check(prm, c, 0, 0, [budget])


@pytest.mark.parametrize("n_units,length", [(1, 150000), (300, 700), (2, 70000)])
def test_evict_cluster_shapes(n_units, length):
    """One long unit on a cluster of eight (more slots a CTA than are held, several rounds of moves), many units on a CTA each."""
    prm = Q.params(n_units, 1, 1, 64, "bf16")
    c = Q.make(prm, np.full(n_units, length) - np.arange(n_units), 64, "bf16", 45)
    scramble(c, 46, ties=n_units == 2)
    evict_and_check_large(prm, c, 4, 100, np.full(n_units, length // 2))


@pytest.mark.parametrize("length", [1500, 9000])
@pytest.mark.parametrize("spread", [1, 40, 3000, 1 << 20])
def test_evict_weights_that_differ_in_their_last_bits(length, spread):
    """A CTA alone and a cluster; every digit of the selection has something to tell, or only the last one."""
    prm = Q.params(4, 1, 1, 64, "bf16")
    c = Q.make(prm, np.full(4, length) - np.arange(4), 32, "bf16", 48)
    r = np.random.default_rng(spread)
    bits = np.float32(0.75).view(np.int32) + r.integers(0, spread, c.mass.numel()).astype(np.int32)
    c.mass.copy_(torch.from_numpy(bits.view(np.float32)).view(c.mass.shape))
    evict_and_check_large(prm, c, 4, 0, [length // 3, 4, length - 5, length // 2])


@pytest.mark.parametrize("length", [1500, 9000])
def test_evict_leaves_exactly_what_has_to_stay(length):
    prm = Q.params(2, 1, 1, 64, "bf16")
    c = Q.make(prm, [length, length - 7], 32, "bf16", 49)
    evict_and_check_large(prm, c, 10, 200, [210, 210])


def evict_and_check_large(prm, c, n_sink, n_recent, budgets):
    """evict_and_check with a sort in place of the oracle's loops, and rows compared on the device."""
    lens, before = Q.lens_of(c), {n: getattr(c, n).clone() for n in ("k", "v", "pos", "mass")}
    B.tca_paged_evict(prm, c, n_sink, n_recent, torch.tensor(np.asarray(budgets), dtype=torch.int32, device="cuda"))
    assert B.tca_paged_status(c)[0] == B.TCA_OK
    mass, pos = before["mass"].cpu().numpy().reshape(-1), before["pos"].cpu().numpy().reshape(-1)
    to, frm = [], []
    for u, n in enumerate(lens):
        rows, budget = Q.pool_rows(c, u, np.arange(n)), int(budgets[u])
        slot = np.arange(n)
        safe = (slot < n_sink) | (pos[rows] > pos[rows].max() - n_recent)
        rank = np.lexsort((slot, -mass[rows].astype(np.float64), ~safe))
        kept = np.zeros(n, dtype=bool)
        kept[rank[:budget]] = True
        to.append(rows[:budget][~kept[:budget]])
        frm.append(rows[budget:][kept[budget:]])
    to, frm = (torch.from_numpy(np.concatenate(x)).cuda() for x in (to, frm))
    for name, x in before.items():
        flat = x.view(-1, prm.head_dim) if name in "kv" else x.view(-1)
        flat[to] = flat[frm]
        assert torch.equal(x, getattr(c, name)), name
    np.testing.assert_array_equal(Q.lens_of(c), np.minimum(lens, budgets))


def test_evict_with_a_page_outside_the_pool_changes_nothing():
    prm = Q.params(2, 1, 1, 64, "bf16")
    c = Q.make(prm, [3000, 500], 32, "bf16", 47)
    c.table[0, 77] = c.n_pages + 3
    before = Q.snapshot(c)
    B.tca_paged_evict(prm, c, 0, 0, torch.tensor([100, 500], dtype=torch.int32, device="cuda"))
    st, detail = B.tca_paged_status(c)
    assert st == B.TCA_ERR_BOUNDS and detail.tolist() == [0, 2]
    before["state"][0, 2] = 2
    Q.same(before, Q.snapshot(c))


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_served_conversation(dtype):
    """Prompts under a window enter the cache with weights, tokens follow one at a time, the cache is cut to its budgets
    again and again and its pages go back to the pool; every result against the oracle over a host copy of what is retained."""
    hq, hkv, d, page, n_sink, n_recent, batch = 8, 2, 64, 16, 2, 8, 3
    prm = Q.params(batch, hq, hkv, d, dtype)
    lens = [90, 37, 150]
    U, G = batch * hkv, hq // hkv
    budgets = np.array([40, 45, 37, 38, 64, 30], dtype=np.int32)
    c = B.PagedCache(prm, 45, page, 12)
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    rows = int(starts[-1])
    q, k, v = (H.packed_buffer(50 + i, h, rows, d, dtype, "tokens") for i, h in enumerate((hq, hkv, hkv)))
    wprm = B.make_params(batch, hq, hkv, d, 32, 33, sm_scale=H.scale_of(d), dtype=H.DC[dtype])
    o, pws = torch.full_like(q, float("nan")), B.alloc_workspace(wprm, rows, B.TCA_OP_PACKED)
    B.tca_attn_window(wprm, q, k, v, rows, torch.from_numpy(starts).cuda(), n_sink, o, pws)
    want, a, s = P.window_attention(H.f64(q), H.f64(k), H.f64(v), starts, 33, n_sink, H.scale_of(d))
    from oracle import serving_oracle as S
    H.check(H.f64(o), want, S.attention_tolerance(want, a, s, d, np.full(want.shape[:2], 150), dtype), "prompts")
    mass = torch.rand(hkv, rows, device="cuda")
    c.reserve(np.repeat(lens, hkv))
    B.tca_paged_append(prm, k, v, rows, starts, None, mass, c)
    host = [dict(k=H.f64(k[u % hkv, starts[u // hkv]:starts[u // hkv + 1]]), v=H.f64(v[u % hkv, starts[u // hkv]:starts[u // hkv + 1]]),
                 pos=np.arange(lens[u // hkv])) for u in range(U)]
    ws, limit = B.alloc_paged_workspace(prm, c, True), torch.from_numpy(budgets).cuda()
    for step in range(24):
        kn, vn, qn = H.randn(100 + step, (hkv, batch, d), dtype), H.randn(200 + step, (hkv, batch, d), dtype), query(prm, 300 + step, dtype)
        if step % 8 == 0:
            m, n = c.mass.cpu().numpy().reshape(-1), Q.lens_of(c)
            src = [P.evict(m[Q.pool_rows(c, u, np.arange(n[u]))], host[u]["pos"], int(budgets[u]), n_sink, n_recent) for u in range(U)]
            B.tca_paged_evict(prm, c, n_sink, n_recent, limit)
            host = [{name: x[src[u]] for name, x in host[u].items()} for u in range(U)]
            c.release(np.minimum(n, budgets))
        c.reserve(np.array([len(h["pos"]) + 1 for h in host]))
        B.tca_paged_append(prm, kn, vn, batch, None, None, None, c)
        o = Q.attend(prm, qn, c, accumulate=True, ws=ws)
        for u in range(U):
            b, h = divmod(u, hkv)
            host[u] = dict(k=np.concatenate([host[u]["k"], H.f64(kn[h, b])[None]]), v=np.concatenate([host[u]["v"], H.f64(vn[h, b])[None]]),
                           pos=np.append(host[u]["pos"], lens[b] + step))
            want, a, s, _ = P.paged_attention(H.f64(qn)[b, h * G:(h + 1) * G], host[u]["k"], host[u]["v"], H.scale_of(d))
            H.check(H.f64(o)[b, h * G:(h + 1) * G], want, P.paged_tolerance(want, a, s, d, 200, dtype), f"step {step} unit {u}")
        snap = Q.snapshot(c)
        for u in range(U):
            r = Q.pool_rows(c, u, np.arange(len(host[u]["pos"])))
            np.testing.assert_array_equal(snap["pos"][r], host[u]["pos"])
            np.testing.assert_array_equal(snap["k"][r], host[u]["k"])
    assert B.tca_paged_status(c)[0] == B.TCA_OK


def test_decode_steps_captured_and_replayed():
    """Append and attend in one graph: the device state moves on with every replay."""
    prm = Q.params(2, 8, 2, 128, "bf16")
    c = Q.make(prm, [100, 100, 31, 31], 32, "bf16", 60, room=20)
    kn, vn, q = H.randn(61, (2, 2, 128), "bf16"), H.randn(62, (2, 2, 128), "bf16"), query(prm, 63, "bf16")
    ws, o = B.alloc_paged_workspace(prm, c, True), torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda")
    limit = torch.tensor([108, 200, 200, 40], dtype=torch.int32, device="cuda")

    def step():
        B.tca_paged_append(prm, kn, vn, 2, None, None, None, c)
        B.tca_attn_paged(prm, q, c, 0, True, o, ws)
        B.tca_paged_evict(prm, c, 1, 2, limit)

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    n0 = Q.lens_of(c)
    for i in range(12):
        kn.copy_(H.randn(70 + i, (2, 2, 128), "bf16"))
        before = Q.snapshot(c)
        g.replay()
        torch.cuda.synchronize()
        assert B.tca_ws_status(ws) == B.TCA_OK and B.tca_paged_status(c)[0] == B.TCA_OK
        # O against the cache as it was after the append: the rows before, and the new one
        for u in range(4):
            b, h = divmod(u, 2)
            n = int(before["state"][u, 0])
            r = Q.pool_rows(c, u, np.arange(n))
            k = np.concatenate([before["k"][r], H.f64(kn[h, b])[None]])
            v = np.concatenate([before["v"][r], H.f64(vn[h, b])[None]])
            want, a, s, _ = P.paged_attention(H.f64(q)[b, h * 4:(h + 1) * 4], k, v, H.scale_of(128))
            H.check(H.f64(o)[b, h * 4:(h + 1) * 4], want, P.paged_tolerance(want, a, s, 128, n + 1, "bf16"), f"replay {i} unit {u}")
    np.testing.assert_array_equal(Q.lens_of(c), np.minimum(n0 + 12, [108, 200, 200, 40]))
