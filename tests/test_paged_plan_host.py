"""How a paged attention call is divided (paged.hpp), computed by the library's own header in a host program."""
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_04511_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

PROGRAM = r'''
#include <cstdio>
#include "paged.hpp"
int main() {
  long long b, h, g, t, k;
  while (std::scanf("%lld %lld %lld %lld %lld", &b, &h, &g, &t, &k) == 5) {
    const sparda::PagedPlan p = sparda::paged_attn_plan((int)b, (int)h, t, (int)k);
    std::printf("%u %d %d %d\n", sparda::paged_units(t, (int)k), p.n_wgs, p.n_splits, sparda::paged_join_waves(p, (int)h, b * h * g));
  }
}
'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("plan")
    src, exe = str(d / "plan.cpp"), str(d / "plan")
    with open(src, "w") as fh:
        fh.write(PROGRAM)
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    src, "-o", exe], check=True)

    def ask(cases):
        out = subprocess.run([exe], input="".join("%d %d %d %d %d\n" % c for c in cases), capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, x.split())) for x in out.splitlines()]
    return ask


CASES = list(itertools.product((1, 2, 8, 16, 32, 64, 200, 700), (1, 2, 8), (1, 4, 16), (1, 64, 1000, 8192, 64000, 2097152),
                               (0, 3, 48, 64, 65, 96, 200, 1000, 32767)))


def test_a_long_row_among_short_ones_is_bounded(plan):
    """Where a row's own workgroups read it and the others may be short, a workgroup has at most 64 units (128 of a list); the
    rest go to the line."""
    for (b, h, g, t, k), (units, n_wgs, n_splits, _) in zip(CASES, plan(CASES)):
        if n_splits < 0:
            assert units <= 16 and n_wgs == -(-b * h // 8), (b, h, t, k)
        elif n_splits > 0:
            assert n_wgs == b * h * n_splits, (b, h, t, k)
            if b > 1:
                assert units <= (128 if k else 64) * n_splits, (b, h, t, k)
        else:
            assert 1 <= n_wgs <= 256 and b > 1, (b, h, t, k)


def test_a_long_row_is_joined_in_few_rounds(plan):
    """All but one sequence may be short: a row of it has then a KV head's share of all workgroups' results, and one more at
    each end.  Up to 1024 (row, head) pairs that takes five rounds at most, up to 16384 nine, more where the pairs keep the chip busy."""
    for (b, h, g, t, k), (_, n_wgs, n_splits, waves) in zip(CASES, plan(CASES)):
        pairs, results = b * h * g, n_splits if n_splits > 0 else n_wgs // h + 2
        if n_splits < 0 or n_splits == 1:
            continue
        rounds = -(-results // (8 * waves))
        assert rounds <= (5 if pairs <= 1024 else 9 if pairs <= 16384 else 33), (b, h, g, t, k)
