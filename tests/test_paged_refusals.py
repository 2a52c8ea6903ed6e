"""Host-side checks of the paged-cache and window entry points (no kernel is launched), the pages a PagedCache deals, and
pins of their oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from oracle import serving_oracle as S
from paper_2512_09238_b200 import _build, binding as B

A = 1 << 20            # an aligned address that nothing dereferences: every call below is refused before a launch


@pytest.fixture(scope="module", autouse=True)
def built_library():
    _build.build()
    return B.lib()


def prm(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=4, head_dim=128, block=32, window=64)
    base.update(kw)
    return B.make_params(**base)


def desc(**kw):
    base = dict(k=A, v=A, pos=A, mass=A, table=A, state=A, n_pages=100, n_units=8, page_size=32, max_pages=20)
    base.update(kw)
    return B.tca_paged_desc(*[base[n] for n, _ in B.tca_paged_desc._fields_])


CALLS = {
    "append": lambda p, d: B.lib().tca_paged_append(C.byref(p), A, A, 2, None, None, None, 2, None, C.byref(d) if d else None, None),
    "attend": lambda p, d: B.lib().tca_attn_paged(C.byref(p), A, C.byref(d) if d else None, 0, 0, A, A, 0, None),
    "evict": lambda p, d: B.lib().tca_paged_evict(C.byref(p), C.byref(d) if d else None, 0, -1, A, None),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_descriptors_are_refused(name):
    call = CALLS[name]
    assert call(prm(), None) == B.TCA_ERR_INVALID_ARG
    for kw in (dict(k=None), dict(v=None), dict(pos=None), dict(mass=None), dict(table=None), dict(state=None), dict(k=A + 8), dict(v=A + 2),
               dict(state=A + 4), dict(table=A + 2), dict(pos=A + 8), dict(mass=A + 4), dict(n_units=7), dict(n_pages=0), dict(max_pages=0)):
        assert call(prm(), desc(**kw)) == B.TCA_ERR_INVALID_ARG, kw
    for kw in (dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(page_size=0), dict(n_pages=1 << 26), dict(max_pages=1 << 26)):
        assert call(prm(), desc(**kw)) == B.TCA_ERR_UNSUPPORTED, kw
    assert call(prm(batch=1 << 14), desc(n_units=1 << 16)) == B.TCA_ERR_UNSUPPORTED
    assert call(prm(batch=1 << 13), desc(n_units=1 << 15, max_pages=1 << 18)) == B.TCA_ERR_UNSUPPORTED     # steps past 32 bits
    for kw in (dict(head_dim=96), dict(n_q_heads=36)):
        assert call(prm(**kw), desc()) == B.TCA_ERR_UNSUPPORTED


def test_attention_refusals():
    p, d = prm(), desc()
    need = B.lib().tca_attn_paged_workspace_bytes(C.byref(p), C.byref(d), 0)
    more = B.lib().tca_attn_paged_workspace_bytes(C.byref(p), C.byref(d), 1)
    assert 0 < need and more == need + 100 * 32 * 2 * 4 + 8 * (20 * 32 // 128 + 2) * 80 + (-8 * 7 * 80) % 256
    assert B.lib().tca_attn_paged_workspace_bytes(C.byref(p), C.byref(desc(page_size=24)), 0) == 0

    def call(p=p, q=A, n_sink=0, acc=0, o=A, ws=A, n=need):
        return B.lib().tca_attn_paged(C.byref(p), q, C.byref(d), n_sink, acc, o, ws, n, None)

    for kw in (dict(q=None), dict(o=None), dict(ws=None), dict(q=A + 8), dict(o=A + 4), dict(ws=A + 128), dict(n_sink=-1)):
        assert call(**kw) == B.TCA_ERR_INVALID_ARG, kw
    assert call(n=need - 1) == call(acc=1, n=more - 1) == B.TCA_ERR_WORKSPACE
    assert call(p=prm(window=0)) == B.TCA_ERR_UNSUPPORTED


def test_append_refusals():
    starts, slots = (C.c_int64 * 3)(0, 10, 90), (C.c_int32 * 2)(0, 1)

    def call(p=None, k=A, v=A, rows=100, strides=None, st=starts, sl=slots, n=2, mass=None):
        s4 = None if strides is None else (C.c_int64 * 4)(*strides)
        return B.lib().tca_paged_append(C.byref(p or prm()), k, v, rows, s4, st, sl, n, mass, C.byref(desc()), None)

    for kw in (dict(k=None), dict(v=None), dict(k=A + 4), dict(v=A + 8), dict(n=3), dict(n=-1), dict(rows=89), dict(rows=-1), dict(rows=1 << 31),
               dict(mass=A + 2), dict(strides=(100, 128, 12800, 128)), dict(strides=(12800, 129, 12800, 128)), dict(strides=(12800, 128, 12800, 1 << 40)),
               dict(sl=(C.c_int32 * 2)(1, 1)), dict(sl=(C.c_int32 * 2)(0, 2)), dict(sl=(C.c_int32 * 2)(-1, 0)), dict(st=(C.c_int64 * 3)(0, 90, 10)),
               dict(st=(C.c_int64 * 3)(-1, 10, 90)), dict(st=None, rows=1)):
        assert call(**kw) == B.TCA_ERR_INVALID_ARG, kw
    assert call(n=0) == B.TCA_OK and call(n=0, st=None) == B.TCA_OK
    assert call(st=(C.c_int64 * 3)(5, 5, 5)) == B.TCA_OK                 # no rows: nothing to do
    assert call(k=None, v=None, rows=0, st=(C.c_int64 * 3)(0, 0, 0)) == B.TCA_OK


def test_evict_refusals():
    def call(d=None, n_sink=0, n_recent=0, budget=A):
        return B.lib().tca_paged_evict(C.byref(prm()), C.byref(d or desc()), n_sink, n_recent, budget, None)
    assert call(n_sink=-1) == call(n_recent=-1) == call(budget=None) == call(budget=A + 2) == B.TCA_ERR_INVALID_ARG
    assert call(d=desc(page_size=256, max_pages=(1 << 14) + 1)) == B.TCA_ERR_UNSUPPORTED      # more than 2^22 slots a unit


def test_window_refusals():
    def call(p=None, n_sink=0, q=A, rows=100, ws_bytes=256, strides=None):
        st = None if strides is None else (C.c_int64 * 8)(*strides)
        return B.lib().tca_attn_window(C.byref(p or prm()), q, A, A, rows, A, st, n_sink, A, A, ws_bytes, None)
    assert call(n_sink=-1) == call(q=None) == call(q=A + 8) == call(rows=-1) == call(strides=[12800, 100] * 4) == B.TCA_ERR_INVALID_ARG
    assert call(p=prm(window=0)) == call(p=prm(head_dim=32)) == B.TCA_ERR_UNSUPPORTED
    assert call(ws_bytes=255) == B.TCA_ERR_WORKSPACE
    assert call(rows=0) == B.TCA_OK


def test_binding_refuses_tensors_that_are_not_on_the_device():
    p = prm()
    c = B.PagedCache(p, 10, 16, 4, device="cpu")
    x, o = torch.zeros(4, 2, 128, dtype=torch.bfloat16), torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    ws = torch.zeros(256, dtype=torch.uint8)
    for call in (lambda: B.tca_paged_append(p, x, x, 2, None, None, None, c), lambda: B.tca_attn_paged(p, o, c, 0, False, o, ws),
                 lambda: B.tca_paged_evict(p, c, 0, 0, torch.zeros(8, dtype=torch.int32)), lambda: B.tca_attn_paged(p, None, c, 0, False, o, ws),
                 lambda: B.tca_paged_append(p, x, x, 2, None, None, None, None),
                 lambda: B.tca_attn_window(p, x, x, x, 2, None, 0, x, ws)):
        with pytest.raises(ValueError):
            call()


def test_pages_are_dealt_and_given_back():
    p = prm()
    c = B.PagedCache(p, 20, 16, 6, device="cpu")
    assert c.state.data_ptr() % 16 == 0 and c.meta.numel() == 2 * 320 + 32
    assert c.mass.dtype == torch.float32 and c.pos.shape == c.mass.shape == (20, 16)
    c.reserve([1, 16, 17, 0, 0, 0, 0, 40])
    assert c.n_held.tolist() == [1, 1, 2, 0, 0, 0, 0, 3] and len(c.free) == 13
    held = c.table_host[c.table_host >= 0]
    assert len(set(held.tolist())) == 7 and not set(held.tolist()) & set(c.free)
    assert (c.table.numpy() == c.table_host).all()
    c.reserve([0] * 8)                                   # never fewer
    assert c.n_held.sum() == 7
    with pytest.raises(B.TcaError):
        c.reserve([97, 0, 0, 0, 0, 0, 0, 0])             # more than max_pages
    with pytest.raises(B.TcaError):
        c.reserve([96, 96, 96, 0, 0, 0, 0, 0])           # more than the pool has
    assert c.n_held.sum() == 7 and len(c.free) == 13
    c.release([0, 16, 16, 0, 0, 0, 0, 33])
    assert c.n_held.tolist() == [0, 1, 1, 0, 0, 0, 0, 3] and len(c.free) == 15 and (c.table.numpy() == c.table_host).all()
    assert (c.table_host[0] == -1).all() and sorted(c.free + c.table_host[c.table_host >= 0].tolist()) == list(range(20))
    for rows in ([1, 2], [-1] + [0] * 7):
        with pytest.raises(ValueError):
            c.reserve(rows)
        with pytest.raises(ValueError):
            c.release(rows)
    with pytest.raises(ValueError):
        B.PagedCache(p, 0, 16, 4, device="cpu")


# ------------------------------------------------------------------ the oracle
def test_window_oracle():
    sees = P.window_mask(6, 2, 1)
    assert sees.astype(int).tolist() == [[1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 1, 1, 0, 0, 0], [1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0],
                                         [1, 0, 0, 0, 1, 1]]
    r = np.random.default_rng(0)
    q, k, v = r.normal(size=(2, 9, 4)), r.normal(size=(1, 9, 4)), r.normal(size=(1, 9, 4))
    for window, sinks in ((9, 0), (1, 9), (100, 3)):
        np.testing.assert_array_equal(P.window_attention(q, k, v, [0, 9], window, sinks, 0.5)[0], S.packed_attention(q, k, v, [0, 9], 0.5)[0])
    np.testing.assert_allclose(P.window_attention(q, k, v, [0, 9], 1, 0, 0.5)[0][0], v[0], rtol=1e-14)


def test_paged_oracle():
    assert P.visible_slots(5, 2, 1).tolist() == [0, 3, 4] and P.visible_slots(0, 3, 2).tolist() == [] and P.visible_slots(3, 9, 0).tolist() == [0, 1, 2]
    r = np.random.default_rng(1)
    q, k, v = r.normal(size=(3, 8)), r.normal(size=(11, 8)), r.normal(size=(11, 8))
    o, _, _, w = P.paged_attention(q, k, v, 0.3)
    p = torch.softmax(torch.from_numpy(q @ k.T * 0.3), -1).numpy()
    np.testing.assert_allclose(o, p @ v, rtol=1e-12)
    np.testing.assert_allclose(w, p.mean(0), rtol=1e-12)
    assert abs(w.sum() - 1) < 1e-12 and P.paged_attention(q, k[:0], v[:0], 0.3)[0].tolist() == np.zeros((3, 8)).tolist()


def test_evict_oracle():
    mass, pos = np.array([0.1, 5, 3, 4, 3, 0]), np.array([0, 7, 2, 3, 9, 8])
    assert P.evict(mass, pos, 6, 0, 0).tolist() == [0, 1, 2, 3, 4, 5]
    assert P.evict(mass, pos, 3, 0, 0).tolist() == [3, 1, 2]             # of the equal slots 2 and 4 the lower one
    assert P.evict(mass, pos, 3, 1, 0).tolist() == [0, 1, 3]
    assert P.evict(mass, pos, 3, 0, 2).tolist() == [4, 1, 5]             # positions 9 and 8 are recent
    assert P.evict(mass, pos, 1, 1, 1) is None and P.evict(mass, pos, 0, 0, 0).tolist() == []
    assert P.evict(np.array([1.0, np.nan, 2.0]), np.arange(3), 1, 0, 0).tolist() == [1]
