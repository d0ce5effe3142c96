"""What the library does on the host for hypotheses and rules, without a GPU:
tests/hip_stub_hypotheses.cpp is linked with the library, stands in for the HIP
calls, makes up the results of the kernels and checks what becomes of them."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

asr = pytest.importorskip("paper_2603_11273_amd.asr")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("stub") / "hypotheses")
    lib_dir = os.path.dirname(asr.LIB_PATH)
    cmd = ["g++", "-std=c++17", "-O1", "-Wall", "-rdynamic", "-I", os.path.join(ROOT, "include"),
           os.path.join(ROOT, "tests", "hip_stub_hypotheses.cpp"), "-L", lib_dir,
           "-l:" + os.path.basename(asr.LIB_PATH), "-Wl,-rpath," + lib_dir,
           "-Wl,--allow-shlib-undefined", "-o", exe]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout

    def run(name):
        r = subprocess.run([exe, name], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
        assert r.returncode == 0, r.stdout[-2000:]
        assert f"{name}: ok" in r.stdout
    return run


def test_a_row_without_a_next_token_ends_its_request_alone(stub):
    """Continuous batching: no allowed token, and a NaN, in one row of two."""
    stub("serve")
