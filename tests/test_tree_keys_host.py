"""Which compressed keys the selection over trees requests (CPU only): with the smallest K~ cache that the call accepts,
every row lies inside it.  tests/host_harness/tree_keys_harness.cpp walks through the requests with the bounds that the
kernel itself uses; the GPU is not involved."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_04511_amd", "csrc")
HARNESS = os.path.join(ROOT, "tests", "host_harness")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, f"{' '.join(cmd[:3])} ... failed ({res.returncode}):\n{res.stdout}\n{res.stderr[-4000:]}"
    return res.stdout


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_selection_reads_inside_the_smallest_key_cache(tmp_path):
    objs = []
    for src in (os.path.join(CSRC, "tree_abi.cpp"), os.path.join(HARNESS, "tree_keys_harness.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        _run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-I", os.path.join(ROOT, "include"),
              "-I", CSRC, "-Wno-unused-function", "-c", src, "-o", objs[-1]])
    exe = str(tmp_path / "tree_keys_harness")
    _run(["g++", *objs, "-o", exe])
    print(_run([exe]))
