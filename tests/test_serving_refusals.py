"""Host-side checks of the serving entry points (no kernel is launched) and pins of their oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

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


def desc(n_units=8, tail_cap=96, ptr=A):
    z = [np.zeros(n_units, dtype=np.int64) for _ in range(7)]
    d = B.tca_cache_desc(ptr, ptr, ptr, ptr, 4096, n_units, tail_cap, *[x.ctypes.data for x in z])
    d.keep_alive = z
    return d


def packed(p, q=A, k=A, v=A, rows=100, start=A, strides=None, o=A, ws=A, ws_bytes=1 << 20):
    st = None if strides is None else (C.c_int64 * 8)(*strides)
    return B.lib().tca_attn_packed(C.byref(p), q, k, v, rows, start, st, o, ws, ws_bytes, None)


def test_packed_refusals():
    p = prm()
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(start=None), dict(o=None), dict(ws=None), dict(q=A + 8),
               dict(o=A + 2), dict(ws=A + 128), dict(start=A + 4), dict(rows=-1), dict(rows=1 << 31)):
        assert packed(p, **kw) == B.TCA_ERR_INVALID_ARG, kw
    good = [12800, 128] * 4
    for i, bad in ((0, 127), (1, 64), (3, 132), (4, -128), (6, 1 << 40), (7, 0)):
        s = list(good)
        s[i] = bad
        assert packed(p, strides=s) == B.TCA_ERR_INVALID_ARG, (i, bad)
    assert packed(p, ws_bytes=255) == B.TCA_ERR_WORKSPACE
    assert packed(p, rows=0) == B.TCA_OK                                # nothing to do
    assert packed(prm(head_dim=96)) == B.TCA_ERR_UNSUPPORTED
    assert packed(prm(n_q_heads=36)) == B.TCA_ERR_UNSUPPORTED           # nine heads per KV head
    assert B.tca_workspace_bytes(p, 100, B.TCA_OP_PACKED) == 256


def test_load_refusals():
    starts, slots = (C.c_int64 * 3)(0, 10, 90), (C.c_int32 * 2)(0, 1)
    def load(p=None, k=A, rows=100, strides=None, st=starts, sl=slots, n=2, d=None):  # noqa: E306
        d = desc() if d is None else d
        s4 = None if strides is None else (C.c_int64 * 4)(*strides)
        return B.lib().tca_cache_load(C.byref(p or prm()), k, A, rows, s4, st, sl, n, C.byref(d), None)
    assert load(k=None) == load(k=A + 4) == load(st=None) == load(n=3) == load(n=-1) == load(rows=89) == B.TCA_ERR_INVALID_ARG
    assert load(strides=(100, 128, 12800, 128)) == load(strides=(12800, 129, 12800, 128)) == B.TCA_ERR_INVALID_ARG
    assert load(sl=(C.c_int32 * 2)(1, 1)) == load(sl=(C.c_int32 * 2)(0, 2)) == B.TCA_ERR_INVALID_ARG
    assert load(st=(C.c_int64 * 3)(0, 90, 10)) == load(d=desc(n_units=6)) == B.TCA_ERR_INVALID_ARG
    assert load(st=(C.c_int64 * 3)(0, 0, 97), rows=97) == B.TCA_ERR_CAPACITY      # a block more than the ring holds
    assert load(d=desc(tail_cap=79)) == B.TCA_ERR_CAPACITY
    assert load(n=0) == B.TCA_OK


def test_no_rows_need_no_buffers():
    assert packed(prm(), q=None, k=None, v=None, o=None, rows=0) == B.TCA_OK
    assert packed(prm(), q=None, k=None, v=None, o=None, rows=0, start=None) == B.TCA_ERR_INVALID_ARG
    d, one = desc(), (C.c_int64 * 1)(0)
    assert B.lib().tca_cache_load(C.byref(prm()), None, None, 0, None, one, None, 0, C.byref(d), None) == B.TCA_OK
    assert B.lib().tca_cache_load(C.byref(prm()), None, None, 1, None, one, None, 0, C.byref(d), None) == B.TCA_ERR_INVALID_ARG


def test_load_finds_a_place_taken_twice_among_many():
    n = 20000
    d = desc(n_units=n, tail_cap=96)
    starts = np.arange(n + 1, dtype=np.int64)
    for a, b in ((0, n - 1), (8191, 8192), (8192, 8193), (16384, 3)):
        slots = np.arange(n, dtype=np.int32)[::-1].copy()
        slots[a] = slots[b]
        assert B.lib().tca_cache_load(C.byref(prm(batch=n, n_q_heads=1, n_kv_heads=1)), A, A, n, None, starts.ctypes.data,
                                      slots.ctypes.data, n, C.byref(d), None) == B.TCA_ERR_INVALID_ARG


def test_load_refuses_starts_that_would_overflow():
    d = desc()
    starts = (C.c_int64 * 2)(1 << 62, -(1 << 62) - 1)
    assert B.lib().tca_cache_load(C.byref(prm()), A, A, 100, None, starts, None, 1, C.byref(d), None) == B.TCA_ERR_INVALID_ARG


def test_tree_refusals():
    def tree(p=None, q=A, kd=A, T=8, parent=A, live=None, d=None, o=A, ws=A, n=1 << 30):
        d = desc() if d is None else d
        return B.lib().tca_attn_tree(C.byref(p or prm()), q, kd, A, T, parent, live, C.byref(d), o, ws, n, None)
    assert tree(q=None) == tree(kd=A + 8) == tree(T=0) == tree(parent=None) == tree(parent=A + 2) == B.TCA_ERR_INVALID_ARG
    assert tree(live=A + 1) == tree(o=None) == tree(ws=A + 16) == tree(d=desc(n_units=4)) == B.TCA_ERR_INVALID_ARG
    assert tree(d=desc(ptr=None)) == tree(d=desc(tail_cap=0)) == B.TCA_ERR_INVALID_ARG
    assert tree(T=129) == B.TCA_ERR_UNSUPPORTED
    p = prm(batch=65536, n_kv_heads=1)
    assert tree(p=p, d=desc(n_units=65536)) == B.TCA_ERR_UNSUPPORTED
    need = B.tca_attn_tree_workspace_bytes(prm(), 8)
    assert need > 256 and tree(n=need - 1) == B.TCA_ERR_WORKSPACE
    assert B.tca_attn_tree_workspace_bytes(prm(), 0) == B.tca_attn_tree_workspace_bytes(prm(), 129) == 0


def test_accept_refusals():
    def accept(p=None, d=None, kd=A, T=8, path=A, n=(1, 2)):
        d = desc() if d is None else d
        na = None if n is None else (C.c_int32 * 2)(*n)
        return B.lib().tca_cache_accept(C.byref(p or prm()), C.byref(d), kd, A, A, T, path, na, None)
    assert accept(kd=None) == accept(kd=A + 8) == accept(T=0) == accept(path=None) == accept(n=None) == B.TCA_ERR_INVALID_ARG
    assert accept(n=(9, 0)) == accept(n=(0, -1)) == accept(d=desc(n_units=2)) == B.TCA_ERR_INVALID_ARG
    assert accept(T=129) == B.TCA_ERR_UNSUPPORTED
    assert accept(d=desc(tail_cap=95)) == B.TCA_ERR_CAPACITY
    d = desc()
    d.keep_alive[4][:] = 95                       # n_tail: the next token fills the ring
    d.keep_alive[6][:] = 4                        # t_keep, with no room in the global region
    assert accept(d=d) == B.TCA_ERR_CAPACITY
    d.keep_alive[4][:] = 96
    assert accept(d=d) == B.TCA_ERR_INVALID_ARG
    assert accept(n=(0, 0)) == B.TCA_OK           # nothing accepted: nothing launched


def test_append_refuses_a_cache_that_16_byte_accesses_cannot_serve():
    def append(d):
        return B.lib().tca_cache_append(C.byref(prm()), C.byref(d), A, A, A, None)
    for off in (2, 4, 8):
        assert append(desc(ptr=A + off)) == B.TCA_ERR_INVALID_ARG
        for field in ("k", "v"):
            d = desc()
            setattr(d, field, A + off)
            assert append(d) == B.TCA_ERR_INVALID_ARG


class OnDevice(torch.Tensor):
    """A host tensor that says it lies on device 0: what the binding looks at before it calls the library."""

    def get_device(self):
        return 0


def test_the_binding_names_what_is_missing_or_no_tensor(monkeypatch):
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    called = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: called.append(name) or 0

    monkeypatch.setattr(B, "_lib", Lib())
    mk = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t).as_subclass(OnDevice)  # noqa: E731
    p = prm(head_dim=64)
    cache = B.Cache(p, np.full(8, 32), 96, np.full(8, 4), device="cpu", init=False)
    cache.k, cache.v = cache.k.as_subclass(OnDevice), cache.v.as_subclass(OnDevice)
    i32, i64 = np.int32, np.int64
    calls = {
        B.tca_attn_packed: dict(Q=mk(8, 10, 64), K=mk(4, 10, 64), V=mk(4, 10, 64), rows=10, seq_start=mk(3, t=torch.int64),
                                O=mk(8, 10, 64), ws=mk(256, t=torch.uint8)),
        B.tca_cache_load: dict(K=mk(4, 10, 64), V=mk(4, 10, 64), rows=10, seq_start=np.array([0, 4, 10], i64),
                               slots=np.array([1, 0], i32), cache=cache),
        B.tca_attn_tree: dict(q=mk(2, 8, 5, 64), k_draft=mk(2, 4, 5, 64), v_draft=mk(2, 4, 5, 64), n_draft=5,
                              parent=mk(2, 5, t=torch.int32), n_live=mk(2, t=torch.int32), cache=cache, O=mk(2, 8, 5, 64),
                              ws=mk(4096, t=torch.uint8)),
        B.tca_cache_accept: dict(cache=cache, k_draft=mk(2, 4, 5, 64), v_draft=mk(2, 4, 5, 64), q_draft=mk(2, 8, 5, 64), n_draft=5,
                                 path=mk(2, 5, t=torch.int32), n_accept=np.array([1, 2], i32)),
    }
    for call, good in calls.items():
        call(p, **good)                                       # the stand-in library takes it
        for name, value in good.items():
            if name in ("rows", "n_draft"):
                continue
            optional = name in ("n_live", "slots")
            for bad in (None, [1, 2, 3], "text", 5, np.zeros((2, 2, 2))):
                if bad is None and optional:
                    call(p, **{**good, name: None})
                    continue
                n = len(called)
                with pytest.raises(ValueError, match=name):
                    call(p, **{**good, name: bad})
                assert len(called) == n
        with pytest.raises(ValueError):
            call(prm(head_dim=64, dtype=7), **good)
    assert len(called) == 6


# ------------------------------------------------------------------ the oracle itself
def test_oracle_paths_of_a_hand_worked_tree():
    sees = S.tree_paths(np.array([-1, 0, 0, 1, -1, 4, 3]))
    assert [list(np.nonzero(r)[0]) for r in sees] == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5], [0, 1, 3, 6]]
    assert [list(np.nonzero(r)[0]) for r in S.tree_paths(np.array([5, 1, -7]))] == [[0], [1], [2]]


def test_oracle_attention_against_closed_forms():
    r = np.random.default_rng(0)
    v = r.normal(size=(6, 4))
    o, a, _ = S.masked_attention(np.zeros((6, 4)), r.normal(size=(6, 4)), v, np.tril(np.ones((6, 6), bool)), 0.5)
    np.testing.assert_allclose(o, np.cumsum(v, 0) / np.arange(1, 7)[:, None])        # equal scores: running means
    np.testing.assert_allclose(a, np.cumsum(np.abs(v), 0) / np.arange(1, 7)[:, None])
    q, k = r.normal(size=(2, 9, 4)), r.normal(size=(1, 9, 4))
    o, _, _ = S.packed_attention(q, k, v[:1].repeat(9, 0)[None], [1, 4, 4, 8], 0.5)  # constant values come back
    assert np.isnan(o[:, [0, 8]]).all()
    np.testing.assert_allclose(o[:, 1:8], np.broadcast_to(v[0], (2, 7, 4)))
    # a chain of drafted tokens over a cache is causal attention over both
    k, v, q = r.normal(size=(9, 4)), r.normal(size=(9, 4)), r.normal(size=(4, 4))
    o, _, _ = S.tree_attention(q, k[:5], v[:5], k[5:], v[5:], np.arange(-1, 3), 0.5)
    vis = np.tril(np.ones((9, 9), bool))[5:]
    np.testing.assert_allclose(o, S.masked_attention(q, k, v, vis, 0.5)[0])


def test_oracle_load_split():
    assert [S.load_split(n, 64, 32) for n in (0, 1, 95, 96, 97, 400)] == [(0, 0), (0, 1), (0, 95), (32, 64), (32, 65), (320, 80)]
