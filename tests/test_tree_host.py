"""The host code of the entry points over trees of drafted tokens under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): compiled host-only with the rest of the library, linked against the stand-in
runtime that checks each launch configuration, and driven by tests/host_harness/tree_harness.cpp."""
import os
import re
import tempfile
from concurrent.futures import ThreadPoolExecutor

from test_host_sanitizers import CLANGXX, CSRC, HARNESS, HIPCC, HOST_FLAGS, LIB_SOURCES, SAN_ENV, _run, tools  # noqa: F401

TREE_SOURCES = ["tree_select.hip", "tree_attention.hip", "tree_verify.hip", "tree_commit.hip", "tree_abi.cpp"]


def test_tree_host_code_under_sanitizers(tools):  # noqa: F811
    with tempfile.TemporaryDirectory() as d:
        srcs = [os.path.join(CSRC, s) for s in LIB_SOURCES + TREE_SOURCES]
        srcs += [os.path.join(HARNESS, "hip_stub.cpp"), os.path.join(HARNESS, "tree_harness.cpp")]
        objs = [os.path.join(d, os.path.basename(s) + ".o") for s in srcs]
        with ThreadPoolExecutor(max_workers=8) as ex:
            list(ex.map(lambda so: _run([HIPCC, *HOST_FLAGS, "-c", so[0], "-o", so[1]]), zip(srcs, objs)))
        fatbins = sorted(set(re.findall(r"\b(__hip_fatbin_\w+)", _run(["nm", "-u", *objs]).stdout)))
        fb = os.path.join(d, "fatbins.cpp")
        with open(fb, "w") as fh:
            fh.writelines(f'extern "C" const char {n}[16] = {{0}};\n' for n in fatbins)
        _run(["g++", "-c", "-fPIC", fb, "-o", fb + ".o"])
        exe = os.path.join(d, "tree_harness")
        _run([CLANGXX, "-fsanitize=address,undefined", *objs, fb + ".o", "-o", exe])
        out = _run([exe], env=SAN_ENV).stdout
        print(out)
        m = re.search(r"(\d+) launches checked, (\d+) with an invalid configuration, (\d+) failed", out)
        assert m and int(m.group(1)) > 1000 and m.group(2) == "0" and m.group(3) == "0"
