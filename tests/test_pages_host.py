"""Page operators without a GPU: what the entry points refuse before anything is launched, the workspace they ask for, and
the host model that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_21603_amd import binding as B
from pages_model import DONE, NONE_LEFT, REFUSED, Model

GOOD = dict(dtype=B.DYN_BF16, n_layers=2, n_kv_heads=2, head_dim=16, page_size=16, n_pages=40, n_rows=6, max_pages_per_row=8, k_cache=0x10000,
            v_cache=0x20000, kv_layer_stride=40 * 1024, block_table=0x30000, seq_len=0x40000, ref_count=0x50000, workspace=0x60000, workspace_bytes=1 << 20)


def pool(**change):
    p = B.dyn_page_pool()
    for name, value in dict(GOOD, **change).items():
        setattr(p, name, value)
    return p


def calls(p):
    a = 0x70000
    lib = B.lib()
    yield "copy", lambda: lib.dyn_pages_copy(C.byref(p), 3, a, a + 64, None)
    yield "fork", lambda: lib.dyn_pages_fork(C.byref(p), 3, a, a + 64, a + 128, None)
    yield "resize", lambda: lib.dyn_pages_resize(C.byref(p), 3, a, a + 64, a + 128, None)
    yield "compact", lambda: lib.dyn_pages_compact(C.byref(p), a, a + 512, None)


@pytest.mark.parametrize("change,status,text", [
    (dict(dtype=5), B.DYN_ERR_INVALID_ARG, "dtype"),
    (dict(n_layers=0), B.DYN_ERR_INVALID_ARG, "non-positive"),
    (dict(n_pages=0), B.DYN_ERR_INVALID_ARG, "non-positive"),
    (dict(page_size=1024), B.DYN_ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=1, head_dim=1, n_kv_heads=1), B.DYN_ERR_UNSUPPORTED, "multiple of 16"),
    (dict(max_pages_per_row=1 << 28), B.DYN_ERR_UNSUPPORTED, "32 bits"),
    (dict(k_cache=None), B.DYN_ERR_INVALID_ARG, "NULL cache"),
    (dict(kv_layer_stride=0), B.DYN_ERR_INVALID_ARG, "kv_layer_stride"),
    (dict(k_cache=0x10008), B.DYN_ERR_INVALID_ARG, "16-byte"),
    (dict(k_cache_layers=0x1000), B.DYN_ERR_INVALID_ARG, "go together"),
])
def test_every_call_refuses_a_pool_that_is_none(change, status, text):
    for name, call in calls(pool(**change)):
        assert call() == status and text in B.dyn_last_error(), (name, B.dyn_last_error())


@pytest.mark.parametrize("change,status,text", [
    (dict(block_table=None), B.DYN_ERR_INVALID_ARG, "NULL table"),
    (dict(ref_count=None), B.DYN_ERR_INVALID_ARG, "NULL table"),
    (dict(workspace=None), B.DYN_ERR_WORKSPACE, "workspace"),
    (dict(workspace=0x60010), B.DYN_ERR_WORKSPACE, "256-byte"),
    (dict(workspace_bytes=64), B.DYN_ERR_WORKSPACE, "needs"),
])
def test_calls_on_tables_refuse_missing_ones(change, status, text):
    for name, call in calls(pool(**change)):
        if name != "copy":
            assert call() == status and text in B.dyn_last_error(), (name, B.dyn_last_error())


def test_missing_and_negative_arguments():
    lib, p = B.lib(), pool()
    assert lib.dyn_pages_copy(C.byref(p), -1, 1, 1, None) == B.DYN_ERR_INVALID_ARG
    assert lib.dyn_pages_copy(C.byref(p), 1, None, 1, None) == B.DYN_ERR_INVALID_ARG
    assert lib.dyn_pages_fork(C.byref(p), 1, 1, 1, None, None) == B.DYN_ERR_INVALID_ARG
    assert lib.dyn_pages_resize(C.byref(p), -2, 1, 1, 1, None) == B.DYN_ERR_INVALID_ARG
    assert lib.dyn_pages_compact(C.byref(p), None, 1, None) == B.DYN_ERR_INVALID_ARG
    assert lib.dyn_pages_copy(None, 1, 1, 1, None) == B.DYN_ERR_INVALID_ARG
    # nothing asked for: nothing launched, nothing read
    assert lib.dyn_pages_copy(C.byref(p), 0, None, None, None) == B.DYN_OK
    assert lib.dyn_pages_fork(C.byref(p), 0, None, None, None, None) == B.DYN_OK
    assert lib.dyn_pages_resize(C.byref(p), 0, None, None, None, None) == B.DYN_OK
    holes = (C.c_void_p * 2)(0x1000, None)
    p = pool(k_cache_layers=C.cast(holes, C.c_void_p), v_cache_layers=C.cast(holes, C.c_void_p))
    assert lib.dyn_pages_copy(C.byref(p), 1, 1, 1, None) == B.DYN_ERR_INVALID_ARG and "layer 1" in B.dyn_last_error()


def test_the_workspace_grows_with_requests_rows_and_pages():
    lib = B.lib()
    size = lambda n, **change: lib.dyn_pages_workspace_bytes(C.byref(pool(**change)), n)
    assert 0 < size(0) <= size(1) < size(1000) and size(0) < size(0, n_pages=4000) and size(0) < size(0, n_rows=4000)
    assert size(-1) == 0 and size(4, dtype=9) == 0


def test_binding_checks_tensors():
    cache = torch.zeros(1, 4, 2, 16, 16)
    table, lens, ref = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for bad in (dict(block_table=table.long()), dict(seq_len=torch.zeros(3, dtype=torch.int32)), dict(ref_count=ref[:3]), dict(block_table=torch.zeros(3, 2, dtype=torch.int32).t()),
                dict(v_cache=torch.zeros(1, 4, 2, 16, 8)), dict(k_cache=cache.half(), v_cache=cache.half())):
        args = dict(dict(k_cache=cache, v_cache=cache, block_table=table, seq_len=lens, ref_count=ref, max_requests=2), **bad)
        with pytest.raises(ValueError):
            B.PagePool(**args)
    with pytest.raises(ValueError, match="on a GPU"):
        B.PagePool(cache, cache, table, lens, ref, 2)


def test_the_model_keeps_counts_in_step_with_rows():
    rs = np.random.RandomState(3)
    k = rs.randn(1, 60, 2)
    m = Model(k, k.copy(), np.zeros((8, 12), np.int32), np.zeros(8, np.int32), np.zeros(60, np.int32), 4)
    seen = set()
    for _ in range(200):
        rows = rs.randint(-1, 9, size=rs.randint(1, 5))
        what = rs.randint(3)
        seen.update(m.resize(rows, rs.randint(0, 50, len(rows))) if what == 0 else m.fork(rs.randint(-1, 9, len(rows)), rows) if what == 1 else [])
        if what == 2:
            m.compact()
        assert np.array_equal(m.counts(), m.ref)
        # a partly filled last page has one owner
        for r, n in enumerate(m.lens):
            if n % 4:
                assert m.ref[m.table[r, n // 4]] == 1
    assert seen == {DONE, NONE_LEFT, REFUSED}
