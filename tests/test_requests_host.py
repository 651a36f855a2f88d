"""libcryptogen_requests.so without a GPU: its host code behind the recording stand-in for the runtime.  What is refused launches
nothing, and no kernel is compiled that no call launches."""
import ctypes as C
import json
import os
import sys

import pytest

from tests.bruteforce import ntt_primes
from tests.stubbed import DEV as d, Stubbed, _Params, run, u32, vp
from workloads.params import PRESETS, ParamSet

u64 = C.c_size_t
KEYS = (vp * 5000)(*[1 << 20] * 5000)
far, farther, at4, odd = vp(1 << 44), vp(1 << 45), vp((1 << 20) + 4), vp((1 << 20) + 2)


class Lib(Stubbed):
    def __init__(self, stub_path, lib_path):
        super().__init__(stub_path, lib_path)
        mine = set(super().compiled())
        self.rq = C.CDLL(os.path.join(os.path.dirname(lib_path), "libcryptogen_requests.so"))
        for name in ("cg_cpvm_requests_workspace_bytes", "cg_cpvm_prepare_workspace_bytes"):
            getattr(self.rq, name).restype = u64
        self.own = [k for k in super().compiled() if k not in mine]

    def handle(self, prm, ctx=None, **change):
        ctx = ctx or self.create(prm)
        q, p = (C.c_uint64 * prm.k)(*prm.q), (C.c_uint64 * prm.nsp)(*prm.p)
        raw, h = _Params(prm.log2n, prm.k, prm.nsp, prm.alpha, prm.t, q, p), vp()
        for name, v in change.items():
            setattr(raw, name, v)
        return self.rq.cg_req_create(C.byref(h), ctx, C.byref(raw)), h


def _calls(n):
    """name -> arguments of a call that is fine (k = 2, N = 4096)"""
    return {
        "cg_slots_encode": [None, d, far, u32(3)],
        "cg_slots_prepare": [None, d, far, u32(3)],
        "cg_cpvm_prepare": [None, d, vp(1 << 28), vp(1 << 29), u32(3), u32(2), u32(100), u32(64), u32(5), far, farther],
        "cg_cpvm_requests": [None, d, d, d, u32(2), at4, u32(3), u32(2), u32(2), u32(64), u32(3), KEYS, KEYS, far, farther],
        "cg_score_bias": [None, d, u32(2), u32(2), u32(2), u32(64), at4, d, at4, u32(3), far],
        "cg_prompt_bias": [None, d, u32(2), u32(2), u32(64), d, at4, u32(3), far],
        "cg_kv_append_requests": [None, far, u32(2), u32(3), u32(2), at4, d, u32(2), d, u32(64)],
    }


# argument -> values that are refused; the numbers are positions after the handle
REFUSED = {
    "cg_slots_encode": {1: [None, at4], 2: [None, d, at4], 3: [u32(0), u32(65537)]},
    "cg_slots_prepare": {1: [None, at4], 2: [None, d, at4], 3: [u32(0), u32(65537)]},
    "cg_cpvm_prepare": {1: [at4, far], 2: [None, at4], 3: [None, at4], 4: [u32(0), u32(65536)], 5: [u32(0)], 6: [u32(0), u32(2049)],
                        7: [u32(0), u32(1), u32(48), u32(2048)], 8: [u32(0), u32(4097)], 9: [None, at4, d], 10: [None, at4, d, far]},
    "cg_cpvm_requests": {1: [None, at4, far], 2: [None, at4], 3: [None, at4], 4: [u32(0), u32(1 << 31)], 5: [None, odd], 6: [u32(0), u32(65536)],
                         7: [u32(0), u32(65536)], 8: [u32(0), u32(3), u32(128)], 9: [u32(0), u32(48), u32(2048)], 10: [u32(8)], 11: [None],
                         12: [None], 13: [None, at4, d], 14: [None, at4, d, far]},
    "cg_score_bias": {1: [None, at4], 2: [u32(0), u32(65536)], 3: [u32(0), u32(65536)], 4: [u32(0), u32(65536)],
                      5: [u32(1), u32(48), u32(2048)], 6: [None, odd], 7: [None, at4], 8: [None, odd], 9: [u32(0), u32(4097)],
                      10: [None, at4, vp((1 << 20) + 4096)]},
    "cg_prompt_bias": {1: [None, at4], 2: [u32(0), u32(65536)], 3: [u32(0), u32(65536)], 4: [u32(1), u32(48), u32(2048)], 5: [None, at4],
                       6: [None, odd], 7: [u32(0), u32(4097)], 8: [None, at4, vp((1 << 20) + 4096)]},
    "cg_kv_append_requests": {1: [None, at4, d], 2: [u32(0)], 3: [u32(0), u32(65536)], 4: [u32(0), u32(65536)], 5: [None, odd],
                              6: [None, at4, far], 7: [u32(0), u32(1)], 8: [None, at4], 9: [u32(0), u32(48), u32(4096)]},
}


def _child(lib):
    from workloads.params import ParamSet
    got = {"accepted": [], "silent": [], "created": {}}
    prm = PRESETS["C1"]
    rc, h = lib.handle(prm)
    assert rc == 0, rc
    f = lib.rq
    for name, args in _calls(prm.n).items():
        assert lib.kernels(lambda: getattr(f, name)(h, *args)), name
        for at, values in REFUSED[name].items():
            for v in values:
                bad = args[:at] + [v] + args[at + 1:]
                lib.stub.stub_log_clear()
                rc = getattr(f, name)(h, *bad)
                if rc != -1 or lib.stub.stub_log_size():
                    got["accepted"].append([name, at, str(v), rc])
        lib.stub.stub_log_clear()
        if getattr(f, name)(None, *args) != -1 or lib.stub.stub_log_size():
            got["accepted"].append([name, "no handle"])
    # a keyless rotation and the parts that may be left out
    keys = (vp * 32)(*[1 << 20] * 31, 0)
    base = _calls(prm.n)
    few = list(base["cg_cpvm_requests"])
    few[11] = (vp * 1)(0)
    got["missing copy key"] = f.cg_cpvm_requests(h, *few)
    few = list(base["cg_cpvm_requests"])
    few[12] = (vp * 30)(*[1 << 20] * 3, 0, *[1 << 20] * 26)
    got["missing block key"] = f.cg_cpvm_requests(h, *few)
    assert f.cg_cpvm_requests(h, None, d, d, None, u32(0), None, u32(1), u32(1), u32(1), u32(64), u32(0), None, KEYS, far, farther) == 0
    assert f.cg_cpvm_prepare(h, None, d, None, None, u32(1), u32(1), u32(100), u32(64), u32(0), far, None) == 0
    assert f.cg_score_bias(h, None, far, u32(1), u32(1), u32(1), u32(64), at4, d, at4, u32(1), far) == 0
    # small arrays that the call would write over while it reads them: within the output or the workspace, to their last entry
    within, last4 = vp(far.value + 64), vp(far.value - 4)
    for name, at, values in (("cg_cpvm_requests", 5, [within, vp(far.value - 8), vp(farther.value + 64)]), ("cg_score_bias", 6, [within, last4]),
                             ("cg_score_bias", 7, [within, vp(far.value - 32)]), ("cg_score_bias", 8, [within, vp(far.value - 8)]),
                             ("cg_prompt_bias", 5, [within]), ("cg_prompt_bias", 6, [within]),
                             ("cg_kv_append_requests", 5, [within, last4]), ("cg_kv_append_requests", 8, [within, vp(far.value - 16)])):
        for v in values:
            bad = base[name][:at] + [v] + base[name][at + 1:]
            lib.stub.stub_log_clear()
            if getattr(f, name)(h, *bad) != -1 or lib.stub.stub_log_size():
                got["accepted"].append([name, at, "overlaps", str(v)])
    # sizes
    got["n_diag"] = [f.cg_cpvm_diagonals(h, u32(a), u32(b)) for a, b in ((1, 64), (768, 64), (2048, 64), (2049, 64), (2048, 128), (2048, 256), (100, 48))]
    assert f.cg_cpvm_requests_workspace_bytes(h, u32(0), u32(1), u32(1)) == f.cg_cpvm_requests_workspace_bytes(h, u32(1), u32(1), u32(0)) == 0
    assert f.cg_cpvm_prepare_workspace_bytes(h, u32(2), u32(100), u32(64), u32(0)) == 0
    assert f.cg_cpvm_prepare_workspace_bytes(h, u32(2), u32(100), u32(64), u32(1)) >= 4 * 2 * 100 * 64
    # scratch of large calls: the units' own ciphertexts, and a bounded part for those that go together
    ws = lambda r, u: f.cg_cpvm_requests_workspace_bytes(h, u32(r), u32(u), u32(1))
    got["ciphertexts a unit beyond"] = (ws(1, 60000) - ws(1, 50000)) / 10000 / (2 * 2 * 4096 * 8)
    assert f.cg_req_destroy(h) == 0 and f.cg_req_destroy(None) == 0
    # creation
    ctx = lib.create(prm)
    for what, change in (("t composite", dict(t=65535)), ("t without slots", dict(t=65521)), ("another ring", dict(log2n=13)),
                         ("fewer primes", dict(k=1)), ("more digits", dict(nsp=2)), ("no primes", dict(q=None))):
        got["created"][what] = lib.handle(prm, ctx, **change)[0]
    got["created"]["t of 40961"] = lib.handle(ParamSet("x", 12, q=prm.q, p=prm.p, t=40961))[0]
    h = vp()
    got["created"]["no context"] = f.cg_req_create(C.byref(h), None, None)
    got["unreached"] = _unreached(lib)
    return got


def _unreached(lib):
    seen, f = set(), lib.rq
    for log2n in (12, 13, 14):
        for k, nsp, alpha in ((1, 1, 1), (2, 1, 1), (3, 1, 1), (6, 2, 2)):
            p = ntt_primes(1 << 50, 2 << log2n, k + nsp)
            rc, h = lib.handle(ParamSet("x", log2n, q=tuple(p[:k]), p=tuple(p[k:]), alpha=alpha))
            assert rc == 0
            go = lambda name, *args: seen.update(x[0] for x in lib.kernels(lambda: getattr(f, name)(h, None, *args)))
            for n in (1, 4, 20, 60, 100, 200, 300, 700):
                b = u32(n)
                go("cg_slots_encode", d, far, b)
                go("cg_slots_prepare", d, far, b)
                go("cg_cpvm_prepare", d, None, None, b, u32(1), u32(100), u32(64), u32(0), far, farther)
                go("cg_cpvm_prepare", None, d, d, b, u32(1), u32(100), u32(64), u32(8), far, farther)
                for d1, n_diag in ((100, f.cg_cpvm_diagonals(h, u32(100), u32(64))), (2048, f.cg_cpvm_diagonals(h, u32(2048), u32(64)))):
                    go("cg_cpvm_requests", d, d, d, u32(2), at4, b, u32(1), u32(n_diag), u32(64), u32(3), KEYS, KEYS, far, farther)
                    go("cg_cpvm_requests", d, d, None, u32(0), None, u32(2), b, u32(n_diag), u32(64), u32(3), KEYS, KEYS, far, farther)
                for d2 in (2, 64, 1024):
                    go("cg_score_bias", d, b, u32(1), u32(1), u32(d2), at4, d, at4, u32(3), far)
                    go("cg_score_bias", far, b, u32(1), u32(1), u32(d2), at4, d, at4, u32(3), far)
                go("cg_kv_append_requests", far, u32(2), b, u32(2), at4, d, u32(2), d, u32(64))
            assert f.cg_req_destroy(h) == 0
    return sorted(set(lib.own) - seen)


@pytest.fixture(scope="module")
def child(tmp_path_factory):
    return run(__file__, tmp_path_factory.mktemp("stub"))


def test_what_is_refused_launches_nothing(child):
    assert child["accepted"] == []
    assert child["missing copy key"] == child["missing block key"] == -1


def test_diagonals_of_a_matrix(child):
    # N = 4096: tiles of 128 (at least N / d2 = 64 and d1), 1024, 2048; none beyond a slot row, or beyond 64 diagonals
    assert child["n_diag"] == [1, 16, 32, 0, 64, 0, 0]


def test_scratch_of_large_calls_is_bounded(child):
    assert child["ciphertexts a unit beyond"] == 1


def test_handles_need_the_contexts_parameters_and_a_modulus_with_slots(child):
    made = child["created"]
    assert made.pop("t of 40961") == 0                       # 1 + 5 * 8192, a prime
    assert set(made.values()) == {-1}, made


def test_every_kernel_is_reached(child):
    assert child["unreached"] == []


def test_alignment_of_the_stand_ins():
    assert d.value % 16 == 0 and at4.value % 16 == 4 and odd.value % 4 == 2


if __name__ == "__main__":
    print(json.dumps(_child(Lib(*sys.argv[1:]))))
