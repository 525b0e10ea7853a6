"""The calls around the paged cache of 4 bits refuse what they cannot take before anything is launched (numbers for pointers: nothing is read), and run on the cache's device."""
import ctypes as C

import pytest
import torch

import test_paged_devices_cpu as devices
from test_paged_devices_cpu import HERE, OTHER, Tensor, ints, lib          # noqa: F401  (lib: a fixture)
from paper_2502_08923_b200 import binding as cs

PTR = 1 << 20


def config(**kw):
    c = cs.CsQuantConfig(PTR, PTR, PTR, PTR, 2 * 16 * 32, 2 * 16 * 2, 10, 16, 2, 64, 0)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def test_workspace_is_host_arithmetic():
    lib = cs.load()
    size = lambda **kw: lib.cs_quant_workspace_bytes(C.byref(config(**kw)))
    sizes = [size(head_dim=d, page_stride=2 * 16 * 64, scale_page_stride=2 * 16 * 4) for d in (32, 64, 128)]
    assert 0 < sizes[0] < sizes[1] < sizes[2] < 64 << 20
    # copies: K and V in 16 bits, of whole sixteens of positions (one of them is always there)
    assert size(tall_positions=1 << 20) - size(tall_positions=1 << 19) == (1 << 19) * 2 * 2 * 64 * 2 + (1 << 15) * 2 * 4 and size(tall_positions=17) == size(tall_positions=32) > size(tall_positions=16) == size()
    assert size(tall_positions=1 << 30) > 1 << 38
    assert lib.cs_quant_workspace_bytes(None) == 0


@pytest.mark.parametrize("field,value,code", [("head_dim", 48, cs.CS_ERR_SHAPE), ("head_dim", 256, cs.CS_ERR_SHAPE), ("head_dim", 0, cs.CS_ERR_SHAPE), ("page_size", 8, cs.CS_ERR_SHAPE), ("page_size", 48, cs.CS_ERR_SHAPE),
                                              ("page_size", -16, cs.CS_ERR_SHAPE), ("n_pages", 0, cs.CS_ERR_ARG), ("n_kv_heads", 0, cs.CS_ERR_ARG), ("page_stride", 1023, cs.CS_ERR_ARG), ("page_stride", 1008, cs.CS_ERR_ARG),
                                              ("page_stride", -1024, cs.CS_ERR_ARG), ("scale_page_stride", 56, cs.CS_ERR_ARG), ("scale_page_stride", 68, cs.CS_ERR_ARG), ("tall_positions", -1, cs.CS_ERR_ARG),
                                              ("tall_positions", (1 << 30) + 1, cs.CS_ERR_ARG), ("k", None, cs.CS_ERR_ARG), ("k", PTR + 8, cs.CS_ERR_ARG), ("v", PTR + 2, cs.CS_ERR_ARG), ("k_scale", None, cs.CS_ERR_ARG),
                                              ("v_scale", PTR + 8, cs.CS_ERR_ARG)])
def test_create_refuses(field, value, code):
    lib, c, h = cs.load(), config(**{field: value}), C.c_void_p()
    assert lib.cs_quant_create(C.byref(h), C.byref(c), PTR, 1 << 50, None) == code
    assert h.value is None and lib.cs_quant_last_error(None).startswith(b"cs_quant_create: ")
    if field not in ("k", "v", "k_scale", "v_scale"):
        assert lib.cs_quant_workspace_bytes(C.byref(c)) == 0


def test_create_refuses_workspaces():
    lib, c, h = cs.load(), config(tall_positions=1000), C.c_void_p()
    n = lib.cs_quant_workspace_bytes(C.byref(c))
    assert lib.cs_quant_create(C.byref(h), C.byref(c), None, n, None) == cs.CS_ERR_ARG
    assert lib.cs_quant_create(C.byref(h), C.byref(c), PTR + 64, n, None) == cs.CS_ERR_ARG
    assert lib.cs_quant_create(C.byref(h), C.byref(c), PTR, n - 1, None) == cs.CS_ERR_CAPACITY
    assert lib.cs_quant_create(None, C.byref(c), PTR, n, None) == cs.CS_ERR_ARG
    assert lib.cs_quant_create(C.byref(h), None, PTR, n, None) == cs.CS_ERR_ARG
    assert lib.cs_quant_create_beside(C.byref(h), C.byref(c), None) == cs.CS_ERR_ARG and lib.cs_quant_last_error(None).startswith(b"cs_quant_create_beside: ")


def test_calls_without_a_handle():
    lib = cs.load()
    assert lib.cs_quant_status(None, None) == cs.CS_ERR_ARG
    assert lib.cs_quant_append(None, None, None, None, None, 0, 0, None, 0, 0, 1e-5, None) == cs.CS_ERR_ARG
    assert lib.cs_quant_read(None, None, None, None, 0, None) == cs.CS_ERR_ARG
    assert lib.cs_quant_attention(None, None, None, 0, 0, 1, 0, 0, 0, 1.0, None, None, None) == cs.CS_ERR_ARG
    assert lib.cs_quant_head_dim(None) == 0 and lib.cs_quant_debug_drop_tile(None, 0) == cs.CS_ERR_ARG
    lib.cs_quant_destroy(None)


def test_pools_that_do_not_fit(monkeypatch):
    pool = lambda *shape, dtype=torch.uint8, cuda=True: type("T", (), dict(is_cuda=cuda, dtype=dtype, device=HERE, shape=torch.Size(shape), dim=lambda s: len(shape), stride=lambda s, d: 1024,
                                                                             __getitem__=lambda s, i: type("U", (), dict(is_contiguous=lambda u: True))()))()
    b = torch.bfloat16
    good = lambda: [pool(10, 2, 16, 32), pool(10, 2, 16, 32), pool(10, 2, 16, 2, dtype=b), pool(10, 2, 16, 2, dtype=b)]
    for i, bad in [(0, pool(10, 2, 16, 32, cuda=False)), (0, pool(10, 2, 16, 32, dtype=torch.int8)), (0, pool(2, 16, 32)), (1, pool(10, 2, 16, 64)), (1, pool(9, 2, 16, 32)), (2, pool(10, 2, 16, 1, dtype=b)),
                   (2, pool(10, 2, 16, 2, dtype=torch.float16)), (3, pool(10, 2, 32, 2, dtype=b))]:
        with pytest.raises(ValueError):
            cs.QuantCache(*(good()[:i] + [bad] + good()[i + 1:]))


def cache(lib):
    c = object.__new__(cs.QuantCache)
    c.lib, c.device, c.head_dim, c.n_kv_heads, c.scale, c.handle, c._id = lib, HERE, 64, 2, 0.125, None, (0, 1)
    return c


READ = dict(block_start=lambda: ints(3), block_len=lambda: ints(3), kv_len=lambda: ints(3), page_table=lambda: ints(3, 7))


@pytest.mark.parametrize("call,arguments", [("cs_quant_attention", devices.ATTENTION), ("cs_quant_append", devices.APPEND), ("cs_quant_read", READ)])
def test_all_on_one_device(lib, call, arguments):          # noqa: F811
    more = dict(out=(Tensor(5, 2, 64), Tensor(5, 2, 64))) if call == "cs_quant_read" else {}
    getattr(cache(lib), call)(**{n: make() for n, make in arguments.items()}, **more)
    assert lib.calls == [(call, HERE)]
    for wrong in arguments:
        given = {n: make() for n, make in arguments.items()}
        given[wrong].device = OTHER
        with pytest.raises(ValueError, match=f"{wrong} is on cuda:0, the call on cuda:1"):
            getattr(cache(lib), call)(**given, **more)
    for i, name in enumerate("kv"):
        if more:
            out = [Tensor(5, 2, 64), Tensor(5, 2, 64)]
            out[i].device = OTHER
            with pytest.raises(ValueError, match=f"{name} is on cuda:0"):
                cache(lib).cs_quant_read(**{n: make() for n, make in arguments.items()}, out=tuple(out))
    assert len(lib.calls) == 1


def test_arguments_that_do_not_fit(lib):                    # noqa: F811
    c, blocks = cache(lib), [make() for make in READ.values()]
    for q in (Tensor(5, 4, 64, dtype=torch.float32), Tensor(5, 4, 32)):
        with pytest.raises(ValueError):
            c.cs_quant_attention(q, *blocks)
    for k, v, kw in ((Tensor(5, 2, 32), Tensor(5, 2, 32), {}), (Tensor(5, 2, 64), Tensor(4, 2, 64), {}), (Tensor(5, 2, 64), Tensor(5, 2, 64), dict(dtype=torch.float32)),
                     (Tensor(5, 2, 64), Tensor(5, 2, 64), dict(q=Tensor(4, 2, 64))), (Tensor(5, 2, 64), Tensor(5, 2, 64), dict(k_gain=Tensor(64, dtype=torch.float32)))):
        with pytest.raises(ValueError):
            c.cs_quant_append(k, v, *blocks, **kw)
    for kw in (dict(), dict(rows=3, dtype=torch.int8), dict(out=(Tensor(5, 2, 64), Tensor(4, 2, 64))), dict(out=(Tensor(5, 3, 64), Tensor(5, 3, 64)))):
        with pytest.raises(ValueError):
            c.cs_quant_read(*blocks, **kw)
    with pytest.raises(ValueError):
        c.cs_quant_attention(Tensor(5, 4, 64), blocks[0], ints(2), *blocks[2:])
    assert not lib.calls
