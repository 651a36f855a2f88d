"""The evaluator alone, and the requests' library with an evaluator that it does not call: programs of their own, no GPU."""
import json
import os
import subprocess
import sys

import pytest

from paper_2602_08798_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import json, os
import paper_2602_08798_amd as P
from paper_2602_08798_amd import binding
lib = P.load_library()
mapped = lambda: "libcryptogen_requests.so" in open("/proc/self/maps").read()
got = {"before": mapped(), "answer": lib.dll.cg_strerror(0) is not None}
try:
    lib.dll.cg_req_create
    got["refused"] = ""
except RuntimeError as e:
    got["refused"] = str(e)
class Context:
    pass
ctx = Context()
ctx.lib, ctx._device_index, ctx.n, ctx.k, ctx.device = lib, 0, 4096, 2, "cuda:0"
if got["refused"]:
    try:
        P.Requests(ctx)
        got["handle"] = ""
    except RuntimeError as e:
        got["handle"] = str(e)
print(json.dumps(got))
"""


def program(**env):
    run = subprocess.run([sys.executable, "-c", PROGRAM], capture_output=True, text=True, cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT, **env})
    assert run.returncode == 0, run.stderr
    return json.loads(run.stdout.splitlines()[-1])


@pytest.fixture
def other_evaluator(tmp_path):
    """a library with the evaluator's entry points, linked without its soname"""
    src, so = tmp_path / "evaluator.c", tmp_path / "evaluator.so"
    src.write_text("".join(f"int {n}(void) {{ return 0; }}\n" for n in binding._SYMBOLS if n != "cg_strerror")
                   + 'const char *cg_strerror(int rc) { (void)rc; return "ok"; }\n')
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)], check=True)
    return str(so)


def test_both_libraries():
    assert program() == {"before": False, "answer": True, "refused": ""}


def test_an_evaluator_without_the_second_library(tmp_path):
    got = program(CRYPTOGEN_REQUESTS_LIB=str(tmp_path / "none.so"))
    assert got["answer"] and "missing" in got["refused"] and got["handle"] == got["refused"]


def test_another_evaluator_runs_and_its_contexts_stay_its_own(other_evaluator):
    got = program(CRYPTOGEN_HIP_LIB=other_evaluator)
    assert got["answer"] and not got["before"]
    assert "another copy" in got["refused"] and got["handle"] == got["refused"]
