"""cs_paged_create_beside refuses what cs_paged_create does, and a first cache that is none (nothing is read or launched)."""
import ctypes as C

import pytest

from paper_2502_08923_b200 import binding as cs
from test_paged_cpu import config


def test_needs_a_first_cache():
    lib, h = cs.load(), C.c_void_p()
    assert lib.cs_paged_create_beside(C.byref(h), C.byref(config()), None) == cs.CS_ERR_ARG
    assert h.value is None and lib.cs_paged_last_error(None).startswith(b"cs_paged_create_beside: ")
    assert lib.cs_paged_create_beside(None, C.byref(config()), None) == cs.CS_ERR_ARG
    assert lib.cs_paged_create_beside(C.byref(h), None, None) == cs.CS_ERR_ARG


@pytest.mark.parametrize("field,value", [("head_dim", 48), ("page_size", 8), ("dtype", 2)])
def test_refuses_configurations(field, value):
    h = C.c_void_p()
    assert cs.load().cs_paged_create_beside(C.byref(h), C.byref(config(**{field: value})), None) == cs.CS_ERR_SHAPE
