"""Attention's choice of tiles and splits (rip_attn_plan.h), built and run on the CPU:
the sizes of attn_plans.py take every variant of the kernels, and every plan covers its
rows within the limits."""
import itertools
import os
import shutil
import subprocess

import pytest

from attn_plans import SHAPES, WIDTHS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "rip_attn_plan.h"
using namespace rip::attn;
static void show(const Plan& p) {
  std::printf("%d %d %d %d %lld ", p.width, p.waves, p.pack, p.splits, (long long)p.slots);
}
int main(int argc, char** argv) {
  for (int i = 1; i + 9 < argc; i += 10) {
    long long v[10];
    for (int j = 0; j < 10; ++j) v[j] = std::atoll(argv[i + j]);
    const Sizes s{v[1], v[2], (int)v[0], (int)v[3], (int)v[4], (int)v[5], v[6] != 0, v[7] != 0, v[8] != 0, (int)v[9]};
    show(plan_forward(s));
    show(plan_dq(s));
    show(plan_dkv(s));
    std::printf("\n");
  }
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
        """(sequences, queries, keys, heads, group, dim, bf16, causal, bias, span) each, in all."""
        args = [str(int(v)) for q in queries for v in q]
        out = subprocess.run([str(d / "p"), *args], capture_output=True, text=True, timeout=60, check=True)
        return [[tuple(int(v) for v in line.split()[5 * i:5 * i + 5]) for i in range(3)]
                for line in out.stdout.splitlines()]
    return run


def test_every_variant_is_taken(plans):
    seen = set()
    cases = list(itertools.product(WIDTHS.items(), (0, 1), (0, 1), SHAPES.values()))
    got = plans([(n, n * q, n * k, heads, group, dim, bf16, causal, bias, 100 * bias)
                 for (width, dim), bf16, bias, (n, q, k, heads, group, causal) in cases])
    for ((width, dim), bf16, bias, shape), plan in zip(cases, got):
        for kind, (w, waves, pack, splits, slots) in zip(("forward", "dq", "dkv"), plan):
            assert w == width
            seen.add((kind, width, bf16, bias, waves, splits > 1))
            if kind != "dkv" and not bias:
                seen.add(("pack", kind, pack > 1))
    for width, bf16, bias, split in itertools.product(WIDTHS, (0, 1), (0, 1), (False, True)):
        eight = bf16 and width in (96, 128)
        for waves in ((4, 8) if eight else (4,)):
            assert ("forward", width, bf16, bias, waves, split) in seen, (width, bf16, bias, waves, split)
        assert ("dq", width, bf16, bias, 8 if eight else 4, split) in seen, (width, bf16, bias, split)
        for waves in ((8,) if eight else (4, 8) if bf16 and width == 64 else (4,)):
            assert ("dkv", width, bf16, bias, waves, split) in seen, (width, bf16, bias, waves, split)
    for kind, packed in itertools.product(("forward", "dq"), (False, True)):
        assert ("pack", kind, packed) in seen


def test_wide_spans_take_four_waves(plans):
    spans = [1, 1468, 1469, 2048]
    for width, dim in WIDTHS.items():
        got = plans([(2, 2000, 2000, 4, 1, dim, 1, 0, 1, s) for s in spans])
        most = 8 if width in (96, 128) else 4
        assert [p[1][1] for p in got] == [most, most, 4, 4]


def test_plans_cover_their_rows(plans):
    sizes = [(n, q, k, heads, group, dim, bf16, causal, bias, span)
             for n in (0, 1, 7, 1 << 20) for q in (0, 1, 130, 70001, 1 << 23) for k in (0, 3, 4097, 1 << 23)
             for heads, group in ((1, 1), (32, 8), (256, 256)) for dim in (1, 64, 96, 250)
             for bf16, causal, bias, span in ((0, 0, 0, 0), (1, 1, 0, 0), (1, 0, 1, 1), (1, 0, 1, 2048))]
    for size, plan in zip(sizes, plans(sizes)):
        n, q, k, heads, group, dim, bf16, causal, bias, span = size
        for kind, (width, waves, pack, splits, slots) in zip(("forward", "dq", "dkv"), plan):
            assert dim <= width and waves in (4, 8) and 1 <= splits <= 64, size
            assert pack == 1 or (pack == group and not bias and kind != "dkv"), size
            # slots for every tile of every sequence, whatever their lengths (and of the
            # tokens before the first and behind the last)
            rows = (k if kind == "dkv" else q) * pack
            assert rows < 1 << 31 and slots == rows // (32 * waves) + n + 2, size


def test_an_empty_side_is_not_split(plans):
    """Nothing to sum into: one part, whatever the other side's length (a second launch over
    no rows would have no workgroups)."""
    sizes = [(n, q, k, heads, group, dim, bf16, causal, bias, bias)
             for n in (0, 1, 7) for q, k in ((0, 128), (0, 600), (0, 100000), (300, 0), (4096, 0), (0, 0))
             for heads, group in ((1, 1), (8, 1), (32, 8)) for dim in (32, 80, 128, 200)
             for bf16 in (0, 1) for causal in (0, 1) for bias in (0, 1)]
    for size, (forward, dq, dkv) in zip(sizes, plans(sizes)):
        assert size[1] or forward[3] == dq[3] == 1, size
        assert size[2] or dkv[3] == 1, size
