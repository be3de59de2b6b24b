"""The weight gradient's choice of tile and split (rip_wgrad_plan.h), built and run on
the CPU: every tile is taken at the sizes of wgrad_tiles.py, which the GPU tests run,
and every plan covers its product."""
import os
import shutil
import subprocess

import pytest

from wgrad_tiles import CASES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "rip_wgrad_plan.h"
using namespace rip::wgrad;
int main(int argc, char** argv) {
  for (int i = 1; i + 3 < argc; i += 4) {
    const int dt = std::atoi(argv[i]);
    const Plan p = make_plan(dt, std::atoll(argv[i + 1]), std::atoll(argv[i + 2]), std::atoll(argv[i + 3]));
    const Shape& s = dt == RIP_BF16 ? kBf16Shapes[p.shape] : kF32Shapes[p.shape];
    std::printf("%d %d %d %d %d %d %lld\n", s.n, s.k, p.tiles_n, p.tiles_k, p.splits, p.part_k,
                (long long)p.share);
  }
  std::printf("%zu %zu\n", sizeof(kF32Shapes) / sizeof(Shape), sizeof(kBf16Shapes) / sizeof(Shape));
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    d = tmp_path_factory.mktemp("plan")
    (d / "p.cpp").write_text(PROGRAM)
    csrc = os.path.join(ROOT, "paper_1909_08029_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    str(d / "p.cpp"), "-o", str(d / "p")], check=True, timeout=120)

    def run(queries):
        args = [str(v) for q in queries for v in q]
        out = subprocess.run([str(d / "p"), *args], capture_output=True, text=True, timeout=60, check=True)
        return [[int(v) for v in line.split()] for line in out.stdout.splitlines()]
    return run


def test_every_tile_is_taken_where_the_gpu_tests_expect_it(plans):
    sizes = [c[0][:3] for c in CASES]
    f32, bf16 = plans([(0, *s) for s in sizes])[:-1], plans([(1, *s) for s in sizes])
    seen = {0: set(), 1: set()}
    for dt, got, at in ((1, bf16, 1), (0, f32, 2)):
        for case, plan in zip(CASES, got):
            assert (tuple(plan[:2]), plan[4] > 1) == case[at], (dt, case[0], plan)
            seen[dt].add(case[at])
    # each tile of the tables, whole and split
    n_f32, n_bf16 = bf16[-1]
    assert len(seen[0]) == 2 * n_f32 and len(seen[1]) == 2 * n_bf16


def test_plans_cover_their_products(plans):
    sizes = [(t, n, k) for t in (0, 1, 31, 32, 33, 257, 4097, 70001, 1 << 23)
             for n in (1, 127, 385, 2048, 1 << 18) for k in (1, 30, 513, 5504, 1 << 18)]
    for dt in (0, 1):
        for (t, n, k), (sn, sk, tn, tk, splits, part_k, share) in zip(sizes, plans([(dt, *s) for s in sizes])):
            assert (tn - 1) * sn < n <= tn * sn and (tk - 1) * sk < k <= tk * sk
            assert share % 32 == 0 and 1 <= splits <= 64
            assert splits * share >= t and (t == 0 or (splits - 1) * share < t)   # none without tokens
            assert part_k % 4 == 0 and 0 <= part_k - k < 4
            assert tn * tk * splits * 512 < 1 << 32                               # a dispatch's work-items
