"""The class Requests without a GPU: what it hands to the entry points, with stand-ins for these and for memory."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_08798_amd import binding, serving
from paper_2602_08798_amd.binding import _REQUEST_SYMBOLS, CgError, Context

N, K = 4096, 2


class Calls:
    """Entry points that answer 0 and keep their arguments; during: what another thread does while one of them runs."""

    def __init__(self):
        self.made, self.during = [], {}

    def __getattr__(self, name):
        def call(*args):
            self.made.append((name, args))
            doing = self.during.pop(name, None)
            if doing:
                doing()
            return {"cg_cpvm_diagonals": 2, "cg_cpvm_prepare_workspace_bytes": 4096, "cg_cpvm_requests_workspace_bytes": 8192}.get(name, 0)
        return call


@pytest.fixture
def requests(monkeypatch):
    """a handle whose tensors are the CPU's"""
    monkeypatch.setattr(serving, "_current_device", lambda: -1)
    monkeypatch.setattr(serving, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 0)
    ctx = object.__new__(Context)
    dll = Calls()
    ctx.lib, ctx.h, ctx.n, ctx.k, ctx._device_index, ctx.device, ctx._ksk_numel = SimpleNamespace(dll=dll), 1, N, K, -1, torch.device("cpu"), 4
    ctx._rounds = {(1, 64, 1): [3, 5]}
    ctx._keys = lambda keys: [k.data_ptr() for k in keys]
    rq = object.__new__(serving.Requests)
    rq.ctx, rq.lib, rq._index, rq.device, rq.n, rq.k, rq._ct, rq.h = ctx, ctx.lib, -1, torch.device("cpu"), N, K, 2 * K * N, 1
    rq._calls = {name: getattr(dll, name) for name in _REQUEST_SYMBOLS}
    rq.dll = dll
    yield rq
    rq.h = ctx.h = None


def prepare(rq):
    rq.cpvm_prepare(1, 100, 64, a=torch.zeros(1, 100, 3, dtype=torch.int64), b=torch.zeros(1, 3, 64, dtype=torch.int64))


def project(rq):
    key = torch.zeros(4, dtype=torch.float64)
    rq.cpvm_requests(torch.zeros(2 * K * N, dtype=torch.int64), torch.zeros(K * N, dtype=torch.float64), 1, 1, 1, 64, [], [key, key])


@pytest.mark.parametrize("name,call", [("cg_cpvm_prepare", prepare), ("cg_cpvm_requests", project)])
def test_calls_made_at_once_have_scratch_of_their_own(requests, name, call):
    """The second call is made while the first one is under way (its entry point lets go of the interpreter): same stream, same handle."""
    requests.dll.during[name] = lambda: call(requests)
    call(requests)
    ws = [args[-1] for made, args in requests.dll.made if made == name]
    assert len(ws) == 2 and 0 not in ws and ws[0] != ws[1]


@pytest.mark.parametrize("closed", ["handle", "context"])
def test_what_is_closed_is_not_asked_anything(requests, closed):
    """No entry point sees a handle whose context is gone: the size of the scratch is asked of both."""
    setattr(requests if closed == "handle" else requests.ctx, "h", None)
    for call in (prepare, project):
        with pytest.raises(CgError):
            call(requests)
    assert {name for name, _ in requests.dll.made} <= {"cg_cpvm_diagonals"}       # (a matter of the ring alone; 0 without a handle)
