"""tca_attn_window against the oracle: window edges, sinks, lengths, layouts, masked garbage, replays, equality with
tca_attn_packed."""
import numpy as np
import pytest
import torch

import serving_harness as H
from oracle import paged_oracle as P
from oracle import serving_oracle as S
from paper_2512_09238_b200 import binding as B

pytestmark = pytest.mark.gpu


def params(n, hq, hkv, d, dtype, window, flags=0):
    return B.make_params(n, hq, hkv, d, 32, window, sm_scale=H.scale_of(d), dtype=H.DC[dtype], flags=flags)


def case(lens, hq, hkv, d, dtype, window, layout="heads", seed=1, lead=3, trail=4, flags=0):
    starts = lead + np.concatenate([[0], np.cumsum(lens)])
    rows = int(starts[-1]) + trail
    mk = lambda i, h: H.packed_buffer(seed + i, h, rows, d, dtype, layout)  # noqa: E731
    return params(len(lens), hq, hkv, d, dtype, window, flags), mk(0, hq), mk(1, hkv), mk(2, hkv), starts


def run(prm, q, k, v, starts, n_sink, out=None, ws=None):
    o = torch.full_like(q, float("nan")) if out is None else out
    ws = B.alloc_workspace(prm, max(1, q.shape[1]), B.TCA_OP_PACKED) if ws is None else ws
    st = torch.tensor(np.asarray(starts), dtype=torch.int64, device="cuda")
    B.tca_attn_window(prm, q, k, v, q.shape[1], st, n_sink, o, ws)
    assert B.tca_ws_status(ws) == B.TCA_OK
    return o


def compare(prm, q, k, v, starts, n_sink, o, dtype):
    want, a, s = P.window_attention(H.f64(q), H.f64(k), H.f64(v), starts, prm.window, n_sink, H.scale_of(prm.head_dim))
    n = np.full(want.shape[:2], max(1, int(np.max(np.diff(starts)))))
    H.check(H.f64(o), want, S.attention_tolerance(want, a, s, prm.head_dim, n, dtype), "window")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (2, 3), (63, 0), (64, 1), (65, 64), (127, 4), (128, 0), (128, 128), (129, 130),
                                           (200, 300), (300, 5), (511, 0), (1000, 7), (1, 1000)])
def test_windows_and_sinks(window, n_sink, dtype):
    prm, q, k, v, starts = case([600, 1, 0, 129, 385], 4, 2, 64, dtype, window)
    compare(prm, q, k, v, starts, n_sink, run(prm, q, k, v, starts, n_sink), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8])
def test_groups(group, dtype):
    prm, q, k, v, starts = case([420, 70, 300], 2 * group, 2, 128, dtype, 100)
    compare(prm, q, k, v, starts, 6, run(prm, q, k, v, starts, 6), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["tokens", "fused", "odd"])
@pytest.mark.parametrize("d", [64, 128])
def test_layouts(layout, d, dtype):
    prm, q, k, v, starts = case([260, 31, 1], 6, 3, d, dtype, 70, layout)
    o = H.packed_buffer(33, 6, q.shape[1], d, dtype, layout)
    o.fill_(float("nan"))
    o = run(prm, q, k, v, starts, 9, out=o)
    compare(prm, q, k, v, starts, 9, o, dtype)


@pytest.mark.parametrize("flags", [0, B.TCA_FLAG_PREFILL_SIMT])
def test_long_prompt(flags):
    """Several items per CTA, many whole tiles; sampled heads."""
    prm, q, k, v, starts = case([4000, 17, 2500], 8, 2, 128, "bf16", 1030, flags=flags)
    o = run(prm, q, k, v, starts, 140)
    sub = [1, 6]
    want, a, s = P.window_attention(H.f64(q[sub]), H.f64(k), H.f64(v), starts, 1030, 140, H.scale_of(128))
    H.check(H.f64(o[sub]), want, S.attention_tolerance(want, a, s, 128, np.full(want.shape[:2], 1200), "bf16"), "long")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 4])
def test_a_window_over_everything_is_the_packed_call(group, dtype):
    for window, n_sink in ((966, 0), ((1 << 31) - 1, 3), (5, 966), (1, (1 << 31) - 1)):
        prm, q, k, v, starts = case([700, 3, 256], 2 * group, 2, 128, dtype, window)
        assert torch.equal(run(prm, q, k, v, starts, n_sink, out=torch.zeros_like(q)),
                           H.run_packed(prm, q, k, v, starts, out=torch.zeros_like(q))), (window, n_sink)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan"), -3.38e38])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,n_sink", [(40, 0), (40, 3), (150, 140), (260, 5)])
def test_hidden_keys_have_no_influence(window, n_sink, dtype, bad):
    """One key and value become infinite, NaN or the lowest number: only the rows that see it may change."""
    L, at = 600, 201
    prm, q, k, v, starts = case([L, 40], 4, 2, 64, dtype, window, lead=0, trail=0)
    clean = run(prm, q, k, v, starts, n_sink)
    k[:, at], v[:, at] = bad, bad
    dirty = run(prm, q, k, v, starts, n_sink)
    sees = P.window_mask(L, window, n_sink)[:, at]
    rows = np.concatenate([np.nonzero(~sees)[0], np.arange(L, L + 40)])
    assert torch.equal(dirty[:, rows], clean[:, rows])
    if not np.isfinite(bad):
        assert not torch.isfinite(dirty[:, np.nonzero(sees)[0]].float()).all(-1).any()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_infinite_values_reach_the_rows_that_see_them(bad):
    """Values alone (keys stay finite): every row that sees the row gets the infinity or NaN in that column only."""
    L, at, col = 500, 130, 17
    prm, q, k, v, starts = case([L], 2, 1, 128, "bf16", 90, lead=0, trail=0)
    clean = run(prm, q, k, v, starts, 0)
    v[:, at, col] = bad
    dirty = run(prm, q, k, v, starts, 0)
    sees = torch.from_numpy(P.window_mask(L, 90, 0)[:, at]).cuda()
    got = dirty[:, :, col].float()
    assert (torch.isnan(got[:, sees]) if np.isnan(bad) else torch.isinf(got[:, sees])).all()
    other = torch.ones(128, dtype=torch.bool, device="cuda")
    other[col] = False
    assert torch.equal(dirty[:, ~sees], clean[:, ~sees]) and torch.equal(dirty[..., other], clean[..., other])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_alone_and_in_a_batch(dtype):
    """The batch around a prompt changes tiles, shapes and orders, not its bits."""
    prm, q, k, v, starts = case([900] + [64] * 5 + [1500] * 8, 8, 4, 64, dtype, 333, lead=0, trail=0)
    whole = run(prm, q, k, v, starts, 70)
    one = params(1, 8, 4, 64, dtype, 333)
    alone = run(one, q[:, :900].contiguous(), k[:, :900].contiguous(), v[:, :900].contiguous(), [0, 900], 70)
    assert torch.equal(whole[:, :900], alone)


def test_replayed_with_other_lengths():
    prm, q, k, v, _ = case([512] * 3, 4, 2, 128, "bf16", 100, lead=0, trail=0)
    st = torch.tensor([0, 512, 1024, 1536], dtype=torch.int64, device="cuda")
    ws, o = B.alloc_workspace(prm, 1536, B.TCA_OP_PACKED), torch.zeros_like(q)
    B.tca_attn_window(prm, q, k, v, 1536, st, 4, o, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        B.tca_attn_window(prm, q, k, v, 1536, st, 4, o, ws)
    for starts in ([0, 512, 1024, 1536], [0, 1, 1400, 1536], [10, 10, 700, 900]):
        st.copy_(torch.tensor(starts, device="cuda"))
        o.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert B.tca_ws_status(ws) == B.TCA_OK
        compare(prm, q, k, v, np.array(starts), 4, o, "bf16")


def test_several_streams_at_once():
    work = []
    for i in range(4):
        prm, q, k, v, starts = case([300 + 50 * i, 40], 4, 2, 128, "bf16", 64 + i, seed=10 * i)
        work.append((prm, q, k, v, starts, torch.full_like(q, float("nan")), B.alloc_workspace(prm, q.shape[1], B.TCA_OP_PACKED),
                     torch.tensor(starts, dtype=torch.int64, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(3):
        for prm, q, k, v, starts, o, ws, st, stream in work:
            with torch.cuda.stream(stream):
                B.tca_attn_window(prm, q, k, v, q.shape[1], st, 5, o, ws)
    torch.cuda.synchronize()
    for prm, q, k, v, starts, o, ws, _, _ in work:
        assert B.tca_ws_status(ws) == B.TCA_OK
        compare(prm, q, k, v, starts, 5, o, "bf16")
