"""The plan of every size that tests/matmul_variants.py is there for, so that a change of the rules
cannot take a kernel out of the GPU tests unseen.  The rules are host code of their own header."""
import os
import subprocess

import pytest

from tests.matmul_variants import VARIANTS, product

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2012_10557_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "matmul_plan.hpp"
int main() {
  long long R, C, T;
  int fp32, dma;
  while (std::scanf("%lld %lld %lld %d %d", &R, &C, &T, &fp32, &dma) == 5) {
    const ekya::MmPlan p = ekya::mm_plan(R, C, T, fp32, dma);
    std::printf("%d %d %d %d %d\n", p.tile, p.splits, p.stages, p.groups, (int)ekya::mm_pack(fp32, R, C, T));
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """plans([(R, C, T, fp32, dma), ..]) -> [(tile, splits, stages, groups, pack), ..]"""
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "plan.cpp", d / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)

    def run(calls):
        text = "\n".join(" ".join(str(int(v)) for v in c) for c in calls)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return run


def test_every_variant_is_reached(plans):
    calls = [(*product(which, *size), prec == "fp32", aligned)
             for _, prec, which, size, aligned, _ in VARIANTS]
    for v, (tile, splits, stages, groups, pack) in zip(VARIANTS, plans(calls)):
        assert (tile, splits, stages, groups) == v[5], v
        assert v[4] or not pack, v  # off 16 bytes, and not copied to it


def test_parts_cover_the_reduction(plans):
    """Stages of all parts reach the sum's end, no part begins behind it, and what a rule may choose
    is what there are kernels for."""
    sizes = [1, 2, 63, 64, 65, 127, 129, 500, 1000, 1500, 2048, 4100, 20000]
    calls = [(R, C, T, f, d) for R in sizes for C in sizes for T in sizes + [100000, 1 << 24]
             for f in (0, 1) for d in (0, 1)]
    for (R, C, T, f, d), (tile, splits, stages, groups, _) in zip(calls, plans(calls)):
        ns = -(-T // (32 if f else 64))
        assert (splits - 1) * stages * groups < ns <= splits * stages * groups, (R, C, T, f, d)
        assert (tile, groups) in ((64, 1), (128, 1), (128, 2), (256, 1))
        assert d and not f or (tile < 256 and groups == 1)
        assert splits <= 512 and (splits == 1 or tile < 256)
