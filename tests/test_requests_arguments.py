"""libcryptogen_requests.so without a GPU: what its kernels are given by calls at the edges of what the header allows."""
import ctypes as C
import json
import os
import subprocess
import sys
from dataclasses import replace

import pytest

from tests.bruteforce import ntt_primes
from tests.stubbed import DEV as d, ROOT, Stubbed, _Params, u32, vp
from workloads.params import PRESETS

far, farther = vp(1 << 44), vp(1 << 45)


class Lib(Stubbed):
    def __init__(self, stub_path, lib_path):
        super().__init__(stub_path, lib_path)
        self.rq = C.CDLL(os.path.join(os.path.dirname(lib_path), "libcryptogen_requests.so"))

    def handle(self, prm, ctx, special=True):
        q, p = (C.c_uint64 * prm.k)(*prm.q), (C.c_uint64 * prm.nsp)(*prm.p)
        raw, h = _Params(prm.log2n, prm.k, prm.nsp, prm.alpha, prm.t, q, p if special else None), vp()
        return self.rq.cg_req_create(C.byref(h), ctx, C.byref(raw)), h

    def arguments(self, count, call):
        """the first `count` arguments of every launch, as int32"""
        self.stub.stub_keep_arguments(count)
        rc = call()
        out = [[self.stub.stub_argument(C.c_size_t(i), a) for a in range(count)] for i in range(self.stub.stub_kept())]
        self.stub.stub_keep_arguments(0)
        assert rc == 0, rc
        return out


def _child(lib):
    got, prm = {"refused": {}, "accepted": []}, PRESETS["C1"]
    ctx = lib.create(prm)
    rc, h = lib.handle(prm, ctx)
    assert rc == 0
    units = 3
    # argument 4 of the low-rank product: how many units share a matrix A
    got["shared"] = {str(group): lib.arguments(5, lambda: lib.rq.cg_cpvm_prepare(
        h, None, None, d, d, u32(units), u32(group), u32(100), u32(64), u32(5), far, farther))[0][4]
        for group in (1, 2, 3, 4, (1 << 31) - 1, 1 << 31, (1 << 32) - 3, (1 << 32) - 1)}
    assert lib.rq.cg_req_destroy(h) == 0
    # parameters of the same sizes that are not the context's
    more = [p for p in ntt_primes(1 << 50, 2 << 12, 9) if p not in prm.q + prm.p]
    q, p = tuple(prm.q), tuple(prm.p)
    for what, other in (("first prime", replace(prm, q=(more[0],) + q[1:])), ("last prime", replace(prm, q=q[:-1] + (more[0],))),
                        ("order of the primes", replace(prm, q=q[::-1])), ("special prime", replace(prm, p=(more[0],))), ("t", replace(prm, t=40961))):
        got["refused"][what] = lib.handle(other, ctx)[0]
    lib.stub.stub_set_device(1)
    got["refused"]["another device"] = lib.handle(prm, ctx)[0]
    lib.stub.stub_set_device(0)
    for special in (True, False):
        rc, h = lib.handle(prm, ctx, special)
        got["accepted"].append(rc)
        lib.rq.cg_req_destroy(h)
    return got


@pytest.fixture(scope="module")
def child(tmp_path_factory):
    from paper_2602_08798_amd import binding
    so = str(tmp_path_factory.mktemp("stub") / "stub.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", so,
                    os.path.join(ROOT, "tests", "host", "hip_arguments_stub.cpp")], check=True)
    run = subprocess.run([sys.executable, os.path.abspath(__file__), so, binding._LIB_PATH], capture_output=True, text=True, cwd=ROOT,
                         env={**os.environ, "PYTHONPATH": ROOT})
    assert run.returncode == 0, run.stderr
    return json.loads(run.stdout)


def test_units_that_share_a_matrix_are_counted_within_32_bits(child):
    """A kernel divides the unit's index by the number: one that passed 31 bits would be below 0 there, and so the index."""
    for group, given in child["shared"].items():
        assert [u // given for u in range(3)] == [u // int(group) for u in range(3)] and given >= 1, (group, given)


def test_a_handle_is_made_for_the_contexts_parameters_on_its_device(child):
    assert set(child["refused"].values()) == {-1}, child["refused"]
    assert child["accepted"] == [0, 0]


if __name__ == "__main__":
    print(json.dumps(_child(Lib(*sys.argv[1:]))))
