"""The paged cache's calls refuse what they cannot take before anything is launched (numbers for pointers: nothing is read)."""
import ctypes as C

import pytest

from paper_2502_08923_b200 import binding as cs

PTR = 1 << 20


def config(**kw):
    c = cs.CsPagedConfig(PTR, PTR, 2 * 16 * 64, 16 * 64, 64, 10, 16, 2, 64, 0)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def test_workspace_is_host_arithmetic():
    lib = cs.load()
    sizes = [lib.cs_paged_workspace_bytes(C.byref(config(head_dim=d, slot_stride=d))) for d in (32, 64, 128)]
    assert 0 < sizes[0] < sizes[1] < sizes[2] < 64 << 20
    assert lib.cs_paged_workspace_bytes(None) == 0


@pytest.mark.parametrize("field,value,code", [("head_dim", 48, cs.CS_ERR_SHAPE), ("head_dim", 256, cs.CS_ERR_SHAPE), ("page_size", 8, cs.CS_ERR_SHAPE), ("page_size", 48, cs.CS_ERR_SHAPE),
                                              ("page_size", -16, cs.CS_ERR_SHAPE), ("dtype", 2, cs.CS_ERR_SHAPE), ("n_pages", 0, cs.CS_ERR_ARG), ("n_kv_heads", 0, cs.CS_ERR_ARG),
                                              ("slot_stride", 60, cs.CS_ERR_ARG), ("slot_stride", 65, cs.CS_ERR_ARG), ("head_stride", 1028, cs.CS_ERR_ARG), ("page_stride", -8, cs.CS_ERR_ARG),
                                              ("k", None, cs.CS_ERR_ARG), ("k", PTR + 8, cs.CS_ERR_ARG), ("v", PTR + 2, cs.CS_ERR_ARG)])
def test_create_refuses(field, value, code):
    lib, c, h = cs.load(), config(**{field: value}), C.c_void_p()
    assert lib.cs_paged_create(C.byref(h), C.byref(c), PTR, 1 << 40, None) == code
    assert h.value is None and lib.cs_paged_last_error(None).startswith(b"cs_paged_create: ")
    if field not in ("k", "v"):
        assert lib.cs_paged_workspace_bytes(C.byref(c)) == 0


def test_create_refuses_workspaces():
    lib, c, h = cs.load(), config(), C.c_void_p()
    n = lib.cs_paged_workspace_bytes(C.byref(c))
    assert lib.cs_paged_create(C.byref(h), C.byref(c), None, n, None) == cs.CS_ERR_ARG
    assert lib.cs_paged_create(C.byref(h), C.byref(c), PTR + 64, n, None) == cs.CS_ERR_ARG
    assert lib.cs_paged_create(C.byref(h), C.byref(c), PTR, n - 1, None) == cs.CS_ERR_CAPACITY
    assert lib.cs_paged_create(None, C.byref(c), PTR, n, None) == cs.CS_ERR_ARG
    assert lib.cs_paged_create(C.byref(h), None, PTR, n, None) == cs.CS_ERR_ARG


def test_calls_without_a_handle():
    lib = cs.load()
    assert lib.cs_paged_status(None, None) == cs.CS_ERR_ARG
    assert lib.cs_paged_append(None, None, None, None, None, 0, None, 0, 0, 1e-5, None) == cs.CS_ERR_ARG
    assert lib.cs_paged_attention(None, None, None, 0, 0, 1, 0, 0, 1.0, None, None, None) == cs.CS_ERR_ARG
    lib.cs_paged_destroy(None)


def test_rows_without_a_context():
    lib = cs.load()
    h = lambda **kw: cs.CsHeads(**(dict(x=PTR, row_stride=512, head_stride=64, y=PTR, y_row_stride=512, y_head_stride=64, n_heads=8) | kw))
    call = lambda q, rows=4, d=64, i=0, o=0, pos=PTR, rope=PTR, n=10, rot=64, eps=1e-5: lib.cs_qk_norm_rope(q, None, rows, d, i, o, pos, rope, n, rot, eps, None)
    assert call(h(), rows=0) == cs.CS_OK and call(h(n_heads=0)) == cs.CS_OK and call(None) == cs.CS_OK
    for bad in (dict(x=None), dict(y=None), dict(x=PTR + 8), dict(y=PTR + 2), dict(gain=PTR + 4), dict(row_stride=516), dict(head_stride=63), dict(y_row_stride=4), dict(n_heads=-1)):
        assert call(h(**bad)) == cs.CS_ERR_ARG, bad
    assert call(h(), rows=-1) == cs.CS_ERR_ARG and call(h(), i=3) == cs.CS_ERR_ARG and call(h(), i=0, o=1) == cs.CS_ERR_ARG and call(h(), i=0, o=2) == cs.CS_ERR_ARG
    assert call(h(), pos=None) == cs.CS_ERR_ARG and call(h(), rope=None) == cs.CS_ERR_ARG and call(h(), n=0) == cs.CS_ERR_ARG and call(h(), eps=-1.0) == cs.CS_ERR_ARG
    assert call(h(), d=48) == cs.CS_ERR_SHAPE and call(h(), rot=24) == cs.CS_ERR_SHAPE and call(h(), rot=128) == cs.CS_ERR_SHAPE and call(h(), rot=-16) == cs.CS_ERR_ARG
    assert lib.cs_rope_table(PTR, 4, 3, 1e4, None) == cs.CS_ERR_ARG and lib.cs_rope_table(PTR, -1, 4, 1e4, None) == cs.CS_ERR_ARG
    assert lib.cs_rope_table(None, 4, 4, 1e4, None) == cs.CS_ERR_ARG and lib.cs_rope_table(PTR, 4, 4, 0.0, None) == cs.CS_ERR_ARG and lib.cs_rope_table(None, 0, 4, 1e4, None) == cs.CS_OK
