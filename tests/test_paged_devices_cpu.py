"""The calls around the paged cache run on the cache's device, and everything they get must be there.  (Stand-ins for tensors of two devices: nothing is launched.)"""
import contextlib

import pytest
import torch

from paper_2502_08923_b200 import binding as cs

HERE, OTHER = torch.device("cuda", 1), torch.device("cuda", 0)


class Tensor:
    """What the binding asks of a tensor."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.bfloat16, device=HERE):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, device

    def dim(self):
        return len(self.shape)

    def stride(self, d):
        n = 1
        for s in self.shape[d + 1:]:
            n *= s
        return n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


class Library:
    """Takes every call down with the device it was made on."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, CURRENT[0]))
            return cs.CS_OK
        return call


CURRENT = [OTHER]


@pytest.fixture
def lib(monkeypatch):
    @contextlib.contextmanager
    def switch(device):
        before, CURRENT[0] = CURRENT[0], device
        yield
        CURRENT[0] = before
    lib = Library()
    monkeypatch.setattr(cs, "load", lambda *a: lib)
    monkeypatch.setattr(cs, "_native", None)
    monkeypatch.setattr(cs, "_stream", lambda: None)
    monkeypatch.setattr(torch.cuda, "device", switch)
    monkeypatch.setattr(torch, "empty", lambda *shape, dtype=None, device=None, **kw: Tensor(*(shape[0] if isinstance(shape[0], torch.Size) else shape), dtype=dtype, device=device))
    return lib


def cache(lib):
    c = object.__new__(cs.PagedCache)
    c.lib, c.k_pages, c.device, c.dtype, c.scale, c.handle, c._id = lib, Tensor(10, 2, 16, 64), HERE, torch.bfloat16, 0.125, None, (0, 0, 1)
    return c


def ints(*shape):
    return Tensor(*shape, dtype=torch.int32)


ATTENTION = dict(q=lambda: Tensor(5, 4, 64), block_start=lambda: ints(3), block_len=lambda: ints(3), kv_len=lambda: ints(3), page_table=lambda: ints(3, 7),
                 out=lambda: Tensor(5, 4, 64), lse=lambda: Tensor(5, 4, dtype=torch.float32))
APPEND = dict(k=lambda: Tensor(5, 2, 64), v=lambda: Tensor(5, 2, 64), block_start=lambda: ints(3), block_len=lambda: ints(3), kv_len=lambda: ints(3), page_table=lambda: ints(3, 7),
              rope=lambda: Tensor(99, 64, dtype=torch.float32), k_gain=lambda: Tensor(64), q=lambda: Tensor(5, 4, 64), q_gain=lambda: Tensor(64), q_out=lambda: Tensor(5, 4, 64))
NORM = dict(q=lambda: Tensor(5, 4, 64), k=lambda: Tensor(5, 2, 64), pos=lambda: ints(5), rope=lambda: Tensor(99, 64, dtype=torch.float32), q_gain=lambda: Tensor(64), k_gain=lambda: Tensor(64))


@pytest.mark.parametrize("call,arguments", [("cs_paged_attention", ATTENTION), ("cs_paged_append", APPEND), ("cs_qk_norm_rope", NORM)])
def test_all_on_one_device(lib, call, arguments):
    f = getattr(cache(lib), call) if call != "cs_qk_norm_rope" else getattr(cs, call)
    f(**{n: make() for n, make in arguments.items()})
    assert lib.calls == [(call, HERE)]                    # not where the caller happens to be
    for wrong in arguments:
        if call == "cs_qk_norm_rope" and wrong == "q":
            continue                                      # (it says where the call is: the others are wrong then)
        given = {n: make() for n, make in arguments.items()}
        given[wrong].device = OTHER
        with pytest.raises(ValueError, match=f"{wrong} is on cuda:0, the call on cuda:1"):
            f(**given)
    assert len(lib.calls) == 1


def test_status_on_the_caches_device(lib):
    assert cache(lib).cs_paged_status() == cs.CS_OK and lib.calls == [("cs_paged_status", HERE)]
