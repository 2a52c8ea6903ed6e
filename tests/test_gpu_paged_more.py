"""Shapes of the paged cache that need many rows or units: evictions of units whose slots do not all fit a CTA's shared memory,
attention whose shares take several rounds of pieces; a status word that changes under running calls; appends of many
CTAs a unit; pages dealt on another stream; a window over an evicted cache."""
import numpy as np
import pytest
import torch

import paged_harness as Q
import serving_harness as H
from paper_2512_09238_b200 import binding as B

pytestmark = pytest.mark.gpu
HELD = 16 * 1024       # slots of a CTA whose weights and positions evict keeps in shared memory


def query(prm, seed, dtype):
    return H.randn(seed, (prm.batch, prm.n_q_heads, prm.head_dim), dtype, 1.5)


# ------------------------------------------------------------------ eviction
def kept_slots(mass, pos, budget, n_sink, n_recent):
    """The definition by one sort: which slots of a unit are kept."""
    slot = np.arange(len(mass))
    safe = (slot < n_sink) | (pos.astype(np.int64) > int(pos.max()) - n_recent)
    assert safe.sum() <= budget
    weight = np.where(np.isnan(mass), np.inf, mass.astype(np.float64))
    rank = np.lexsort((slot, -weight, ~np.isnan(mass), ~safe))
    kept = np.zeros(len(mass), dtype=bool)
    kept[rank[:budget]] = True
    return kept


def evict_and_check(prm, c, n_sink, n_recent, budgets):
    lens, before = Q.lens_of(c), {n: getattr(c, n).clone() for n in ("k", "v", "pos", "mass")}
    B.tca_paged_evict(prm, c, n_sink, n_recent, torch.tensor(np.asarray(budgets), dtype=torch.int32, device="cuda"))
    assert B.tca_paged_status(c)[0] == B.TCA_OK
    mass, pos = before["mass"].cpu().numpy().reshape(-1), before["pos"].cpu().numpy().reshape(-1)
    to, frm = [], []
    for u, n in enumerate(lens):
        budget = int(budgets[u])
        if n <= budget:
            continue
        rows = Q.pool_rows(c, u, np.arange(n))
        kept = kept_slots(mass[rows], pos[rows], budget, n_sink, n_recent)
        to.append(rows[:budget][~kept[:budget]])
        frm.append(rows[budget:][kept[budget:]])
    to, frm = (torch.from_numpy(np.concatenate(x)).cuda() for x in (to, frm))
    for name, x in before.items():
        flat = x.view(-1, prm.head_dim) if name in "kv" else x.view(-1)
        flat[to] = flat[frm]
        a, b = (t.view(torch.int32) if name == "mass" else t for t in (x, getattr(c, name)))
        assert torch.equal(a, b), name
    np.testing.assert_array_equal(Q.lens_of(c), np.minimum(lens, budgets))


def weigh(c, seed, kind):
    """Positions in no order; weights: "distinct", "ties" (few values) or "nans" (some of them NaN, in many ties)."""
    r = np.random.default_rng(seed)
    pos, mass = c.pos.cpu().numpy().reshape(-1), c.mass.cpu().numpy().reshape(-1)
    for u, n in enumerate(Q.lens_of(c)):
        n, rows = int(n), Q.pool_rows(c, u, np.arange(n))
        pos[rows] = r.permutation(2 * n)[:n]
        mass[rows] = r.permutation(n) * 0.25 + 1 if kind == "distinct" else r.integers(0, 5, n)
        if kind == "nans":
            mass[rows[r.random(n) < 0.3]] = np.nan
    c.pos.copy_(torch.from_numpy(pos).view(c.pos.shape))
    c.mass.copy_(torch.from_numpy(mass).view(c.mass.shape))


@pytest.mark.parametrize("kind", ["distinct", "ties", "nans"])
def test_evict_one_unit_of_more_slots_than_a_cluster_holds(kind):
    """A cluster of 16 CTAs at most; every CTA reads the slots behind its first 16384 again at each pass."""
    n = 16 * HELD + 16 * 700 + 3
    prm = Q.params(1, 1, 1, 64, "bf16")
    c = Q.make(prm, [n], 64, "bf16", 60)
    weigh(c, 61, kind)
    evict_and_check(prm, c, 5, 300, [n // 2 + 1])        # several rounds of moves
    weigh(c, 62, kind)
    evict_and_check(prm, c, 5, 300, [n // 7])


@pytest.mark.parametrize("kind", ["distinct", "ties", "nans"])
def test_evict_units_of_more_slots_than_a_cta_holds(kind):
    """So many units that each has one CTA, a few of them longer than its shared memory."""
    U = 2 * torch.cuda.get_device_properties(0).multi_processor_count + 4
    lens = np.full(U, 5)
    lens[[0, 7, U // 2, U - 1]] = [HELD, HELD + 1, 2 * HELD + 4099, HELD + 62]
    prm = Q.params(U, 1, 1, 64, "f32")
    c = Q.make(prm, lens, 32, "f32", 63)
    weigh(c, 64, kind)
    evict_and_check(prm, c, 3, 50, np.where(lens > 5, lens // 2 - 1, 5))


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("dtype,hq,d", [("bf16", 2, 64), ("bf16", 8, 128), ("f32", 1, 64), ("f32", 2, 64), ("f32", 5, 128)])
def test_several_rounds_of_pieces_with_units_across_shares(dtype, hq, d):
    """More than 128 pieces in every share (one round of the list), and units that run from one share into others."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    n = 140 * sms + 11
    prm = Q.params(n, hq, 1, d, dtype)
    r = np.random.default_rng(hq)
    lens = r.integers(1, 16, n)
    lens[r.permutation(n)[:6]] = [30000, 25000, 40001, 127, 2000, 33000]
    c = Q.make(prm, lens, 16, dtype, 70)
    q, ws = query(prm, 71, dtype), B.alloc_paged_workspace(prm, c, True)
    o = Q.attend(prm, q, c, ws=ws)
    Q.check(prm, q, c, o, 0, dtype)
    before = Q.snapshot(c)
    Q.check(prm, q, c, Q.attend(prm, q, c, accumulate=True, ws=ws), 0, dtype, before)
    assert torch.equal(o, Q.attend(prm, q, c, ws=ws))


@pytest.mark.parametrize("accumulate", [False, True])
def test_a_status_word_that_changes_under_running_calls(accumulate):
    """Somebody else sets and clears the status word all the time: every call still ends, writes nothing but its results, and
    the zeroed workspace is as good as new."""
    prm = Q.params(6, 8, 2, 128, "bf16")
    c = Q.make(prm, [30000, 20, 700, 9000, 0, 1, 130, 260, 5000, 3, 64, 12000], 32, "bf16", 90)
    ws, q = B.alloc_paged_workspace(prm, c, accumulate), query(prm, 91, "bf16")
    good, before = Q.attend(prm, q, c, ws=ws), Q.snapshot(c)
    words = [torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")]
    o, status, side = torch.empty_like(q), ws[:4].view(torch.int32), torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(300):
        B.tca_attn_paged(prm, q, c, 0, accumulate, o, ws)
        with torch.cuda.stream(side):
            for j in range(6):
                status.copy_(words[j & 1])
    torch.cuda.synchronize()
    Q.same(before, Q.snapshot(c), ("mass",) if accumulate else ())
    ws.zero_()
    assert torch.equal(good, Q.attend(prm, q, c, ws=ws))


def test_append_with_many_ctas_a_unit_again_and_again():
    """Up to 40 CTAs read a unit's length before the last of them moves it on; ten calls in a row, the same ones replayed."""
    prm = Q.params(4, 3, 3, 64, "bf16")
    new, again = np.array([5000, 129, 700, 2561]), 10
    c = Q.make(prm, np.zeros(12), 64, "bf16", 95, room=int(new.max()) * 2 * again)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    rows = int(starts[-1])
    k, v = (H.packed_buffer(96 + i, 3, rows, 64, "bf16", "tokens") for i in range(2))
    calls = lambda: [B.tca_paged_append(prm, k, v, rows, starts, None, None, c) for _ in range(again)]  # noqa: E731
    calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        calls()
    g.replay()
    torch.cuda.synchronize()
    assert B.tca_paged_status(c)[0] == B.TCA_OK
    state = c.state.cpu().numpy().reshape(4, 3, B.TCA_PG_STATE_WORDS)
    for word in (B.TCA_PG_LEN, B.TCA_PG_NEXT):
        np.testing.assert_array_equal(state[:, :, word], np.repeat(2 * again * new[:, None], 3, 1))
    assert (state[:, :, 3] == 0).all()
    for s, n in enumerate(new):
        for h in range(3):
            r = torch.from_numpy(Q.pool_rows(c, s * 3 + h, np.arange(2 * again * n))).cuda()
            part = slice(int(starts[s]), int(starts[s + 1]))
            for pool, x in ((c.k, k), (c.v, v)):
                assert torch.equal(pool.view(-1, 64)[r].view(2 * again, int(n), 64), x[h, part].expand(2 * again, -1, -1))
            assert torch.equal(c.pos.view(-1)[r].long().cpu(), torch.arange(2 * again * int(n)))


def test_pages_change_hands_on_the_stream_of_the_calls():
    """A call that waits in its stream reads the pages it was given, although they are dealt anew behind it."""
    prm = Q.params(2, 4, 2, 64, "bf16")
    c = Q.make(prm, [300, 40, 500, 129], 32, "bf16", 97, max_pages=20, spare=0)
    q, ws = query(prm, 98, "bf16"), B.alloc_paged_workspace(prm, c)
    want, o, side = Q.attend(prm, q, c, ws=ws), torch.full_like(q, float("nan")), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)                   # 0.1 s
    B.tca_attn_paged(prm, q, c, 0, False, o, ws, stream=side)
    c.release([0, 0, 0, 0], stream=side)
    assert (c.table_host == -1).all()
    c.reserve([0, 600, 0, 1], stream=side)
    with torch.cuda.stream(side):
        c.state.zero_()
    k, v = (H.randn(99 + i, (2, 2, 64), "bf16") for i in range(2))
    torch.cuda.current_stream().synchronize()
    c.reserve([1, 0, 1, 0], stream=side)
    B.tca_paged_append(prm, k, v, 2, None, None, None, c, stream=side)
    side.synchronize()
    assert B.tca_ws_status(ws) == B.TCA_OK and B.tca_paged_status(c)[0] == B.TCA_OK
    assert torch.equal(o, want)
    np.testing.assert_array_equal(c.table.cpu().numpy(), c.table_host)
    for u in range(4):
        assert torch.equal(c.k.view(-1, 64)[Q.pool_rows(c, u, [0])[0]], k[u % 2, u // 2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_window_over_an_evicted_cache_goes_by_slots(dtype):
    """What stays visible are the last slots and the sinks, whatever positions their rows have; a window that hides nothing sees
    every row that was kept."""
    prm = Q.params(2, 4, 2, 64, dtype, window=20)
    c = Q.make(prm, [300, 700, 41, 260], 32, dtype, 92)
    B.tca_paged_evict(prm, c, 4, 30, torch.tensor([120, 200, 60, 90], dtype=torch.int32, device="cuda"))
    assert B.tca_paged_status(c)[0] == B.TCA_OK and Q.lens_of(c).tolist() == [120, 200, 41, 90]
    pos = c.pos.cpu().numpy().reshape(-1)
    assert pos[Q.pool_rows(c, 1, np.arange(180))].max() >= 670       # recent rows lie where the window hides them
    for p in (prm, Q.params(2, 4, 2, 64, dtype)):
        q, before = query(prm, 93, dtype), Q.snapshot(c)
        Q.check(p, q, c, Q.attend(p, q, c, 4, accumulate=True), 4, dtype, before)
