"""The sizes that include/tca.h says the paged cache supports, at their edges (host checks; no kernel is launched)."""
import ctypes as C

import pytest

from paper_2512_09238_b200 import _build, binding as B

A = 1 << 20            # an aligned address that nothing dereferences


@pytest.fixture(scope="module", autouse=True)
def built_library():
    _build.build()
    return B.lib()


def supported(units, n_pages, page_size, max_pages):
    """Whether the paged calls take such a cache: the workspace size is 0 for those that they refuse."""
    p = B.make_params(batch=units, n_q_heads=2, n_kv_heads=1, head_dim=64, block=32, window=64)
    d = B.tca_paged_desc(A, A, A, A, A, A, n_pages, units, page_size, max_pages)
    size = B.lib().tca_attn_paged_workspace_bytes(C.byref(p), C.byref(d), 0)
    st = B.lib().tca_attn_paged(C.byref(p), A, C.byref(d), 0, 0, A, A, 0, None)       # too small a workspace, if nothing else
    assert st == (B.TCA_ERR_WORKSPACE if size else B.TCA_ERR_UNSUPPORTED)
    return size > 0


def test_pool_and_table():
    assert supported(1, (1 << 27) - 1, 16, 4) and not supported(1, 1 << 27, 16, 4)
    assert supported(1, 4, 16, (1 << 27) - 17) and not supported(1, 4, 16, (1 << 27) - 16)
    assert supported(65535, 4, 256, 4) and not supported(65536, 4, 256, 4)


def test_steps_of_all_units():
    """128 units of 2^31 - 512 slots are 128 (2^24 - 1) steps; one more unit is too much."""
    assert supported(128, 4, 256, (1 << 23) - 2) and not supported(129, 4, 256, (1 << 23) - 2)
    slots = 1 << 22
    most = ((1 << 31) - 1) // (slots // 128 + 3)
    assert most < 65535 and supported(most, 4, 256, slots // 256) and not supported(most + 1, 4, 256, slots // 256)


def test_eviction_takes_fewer_slots_a_unit():
    p = B.make_params(batch=1, n_q_heads=1, n_kv_heads=1, head_dim=64, block=32, window=64)
    d = B.tca_paged_desc(A, A, A, A, A, A, 4, 1, 256, (1 << 14) + 1)       # 2^22 slots and a page
    assert B.lib().tca_paged_evict(C.byref(p), C.byref(d), 0, 0, A, None) == B.TCA_ERR_UNSUPPORTED
    assert B.lib().tca_attn_paged(C.byref(p), A, C.byref(d), 0, 0, A, A, 0, None) == B.TCA_ERR_WORKSPACE     # attention does not mind
