"""The paged cache's refusals that need no device."""
import ctypes as C

import paper_2510_14961_b200 as rd
from paper_2510_14961_b200 import binding


def _config(**kw):
    base = dict(n_heads=4, n_kv_heads=2, head_dim=64, dtype=rd.RD_BF16, page_size=16, n_pages=4, n_layers=1, max_context=64, max_rows=0,
                rope_base=10000.0)
    base.update(kw)
    return binding.RdPagedConfig(**base)


def test_configurations_that_are_refused():
    L, out = rd.lib(), C.c_void_p()
    assert L.rd_paged_create(None, None, None, C.byref(out)) == rd.RD_E_INVALID_ARG
    assert L.rd_paged_create(C.byref(_config()), None, None, None) == rd.RD_E_INVALID_ARG
    assert L.rd_paged_create(C.byref(_config()), 4096, None, C.byref(out)) == rd.RD_E_INVALID_ARG       # one pool of two
    assert L.rd_paged_create(C.byref(_config()), 4096 + 8, 8192, C.byref(out)) == rd.RD_E_INVALID_ARG   # not aligned
    assert L.rd_paged_create(C.byref(_config()), 1 << 20, (1 << 20) + 4096, C.byref(out)) == rd.RD_E_INVALID_ARG   # overlapping
    for kw in (dict(n_heads=0), dict(n_heads=5), dict(n_kv_heads=0), dict(head_dim=0), dict(head_dim=7), dict(head_dim=130), dict(dtype=5),
               dict(page_size=0), dict(page_size=8), dict(page_size=17), dict(page_size=512), dict(n_pages=0), dict(n_layers=-1),
               dict(max_context=0), dict(max_rows=-5), dict(rope_base=-1.0), dict(rope_base=float("nan")), dict(rope_base=float("inf"))):
        assert L.rd_paged_create(C.byref(_config(**kw)), None, None, C.byref(out)) == rd.RD_E_INVALID_ARG, kw
    assert L.rd_paged_create(C.byref(_config(n_pages=1 << 30)), None, None, C.byref(out)) == rd.RD_E_CAPACITY
    assert L.rd_paged_create(C.byref(_config(max_rows=1 << 30)), None, None, C.byref(out)) == rd.RD_E_CAPACITY
    assert L.rd_paged_create(C.byref(_config(max_context=(1 << 30) + 1)), None, None, C.byref(out)) == rd.RD_E_CAPACITY
    assert not out


def test_null_arguments():
    L, rows = rd.lib(), binding.RdPagedRows()
    assert L.rd_paged_append(None, C.byref(rows), 0, *([None, 0] * 4), None) == rd.RD_E_INVALID_ARG
    assert L.rd_paged_attend(None, C.byref(rows), 0, None, 0, None, 0, None, 0, 0, C.c_float(0), None) == rd.RD_E_INVALID_ARG
    assert L.rd_paged_sync(None, None) == rd.RD_E_INVALID_ARG
    assert L.rd_paged_pages(None, None, None) == rd.RD_E_INVALID_ARG
    L.rd_paged_destroy(None)
