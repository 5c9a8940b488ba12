"""The plan of a layer with block scales (csrc/w4a8_blocks_plan.h), compiled with the host compiler: it fits the hardware for any
size, deals the channels out without a CTA that has none, and takes the kernel for which a test shape is there."""
import os
import random
import subprocess

import pytest

from blocks_shapes import EXPERTS_FEW, EXPERTS_MANY, EXPERTS_MANY_LAYERS, FEW, MANY

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = r"""
#include <cstdio>
#include "w4a8_blocks_plan.h"
using namespace w4a8;
int main() {
    long long rows, experts, N, K, sms, grouped;
    while (std::scanf("%lld %lld %lld %lld %lld %lld", &rows, &experts, &N, &K, &sms, &grouped) == 6) {
        const BlocksPlan p = blocks_plan(rows, experts, N, K, (int)sms, grouped != 0);
        const BlocksSmem s = blocks_smem(p.tmax, p.channels, p.tokens, p.stages, p.cut, p.share, p.part_buffers, grouped != 0);
        std::printf("%d %d %d %d %d %d %d %d %d %d %lld %d %d %d %d %d\n", p.wide, p.tmax, p.tokens, p.channels, p.cut, p.share, p.part_buffers,
                    p.stages, p.smem, p.ctas, (long long)p.tiles, s.bars, s.scales, s.table, s.parts, s.end);
    }
}
"""
NAMES = "wide tmax tokens channels cut share part_buffers stages smem ctas tiles bars scales table parts end".split()


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SRC)
    exe = str(d / "plan")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2505_14638_b200", "csrc"),
                    "-o", exe, str(d / "plan.cpp")], check=True)

    def ask(cases):
        text = "".join("%d %d %d %d %d %d\n" % c for c in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        return [dict(zip(NAMES, map(int, line.split()))) for line in out]
    return ask


def _check(p, rows, experts, N, K, sms, grouped):
    kb = -(-K // 128)
    if p["wide"]:
        assert p["tokens"] == 128 and rows > 64 and N > 128
        return
    assert p["tmax"] in (16, 32, 64, 128) and 16 <= p["tokens"] <= p["tmax"] and p["tokens"] % 16 == 0
    assert p["channels"] % 8 == 0 and 64 <= p["channels"] <= 128
    assert 1 <= p["cut"] <= 8 and p["cut"] <= kb
    assert p["ctas"] == (2 if p["tmax"] <= 32 else 1)
    # every CTA of a cluster writes at least eight channels, none more than there is room for
    units = p["channels"] // 8
    first = [r * units // p["cut"] for r in range(p["cut"] + 1)]
    assert all(8 <= 8 * (b - a) <= p["share"] for a, b in zip(first, first[1:])) and p["share"] % 8 == 0
    for u in range(units):
        owner = ((u + 1) * p["cut"] - 1) // units
        assert first[owner] <= u < first[owner + 1]
    # a ring of four stages at least, its parts one behind the other, and all of it within the SM
    stage = p["channels"] * 128 + -(-p["tokens"] // 32) * 4096
    assert 4 <= p["stages"] <= 16 and p["bars"] == p["stages"] * stage
    assert p["scales"] >= p["bars"] + 8 * (2 * 16 + 2 * 4 + 2 + 2 + 1) + 8 and p["scales"] % 16 == 0
    assert p["table"] >= p["scales"] + 2 * 2 * 8 * p["tmax"] * 4 and p["table"] % 16 == 0
    assert p["parts"] >= p["table"] + (2 * 513 * 4 + 32 if grouped else 0) and p["parts"] % 16 == 0
    assert p["end"] >= p["parts"] + p["part_buffers"] * p["cut"] * p["tokens"] * p["share"] * 4
    assert p["end"] >= (p["stages"] - 1) * stage + 128 * 128          # what the last stage's MMA reads
    assert p["smem"] == 1024 + p["end"] <= (232448 if p["ctas"] == 1 else 115712)
    # one tile of tokens covers a layer's tokens, or several do
    if experts == 1:
        assert p["tiles"] == -(-N // p["channels"]) * -(-rows // p["tokens"])


def test_any_size_has_a_plan(plan):
    r = random.Random(7)

    def size(lo, hi, mult):
        return max(mult, int(2 ** r.uniform(lo, hi)) // mult * mult)
    cases = []
    for _ in range(6000):
        experts = r.choice([1, 1, 2, 8, 40, 128, 512])
        cases.append((size(0, 18, 1), experts, size(4, 16, 16), size(4, 16, 16), r.choice([148, 148, 132, 160, 8]), int(experts > 1 or r.random() < 0.3)))
    for m in (1, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 2 ** 30):
        cases += [(m, 1, 16, 16, 148, 0), (m, 1, 65552, 65536, 148, 0), (m, 512, 4096, 4096, 148, 1)]
    plans = plan(cases)
    assert len(plans) == len(cases)
    for c, p in zip(cases, plans):
        _check(p, *c)
    assert {p["cut"] for p in plans if not p["wide"]} == set(range(1, 9))


def test_the_shapes_of_the_gpu_tests_reach_both_kernels(plan):
    for shapes, wide in ((FEW, 0), (MANY, 1)):
        for s, p in zip(shapes, plan([(M, 1, N, K, 148, 0) for M, N, K in shapes])):
            assert p["wide"] == wide, s
    for counts in EXPERTS_FEW:
        for p in plan([(sum(counts) + 6, len(counts), N, K, 148, 1) for N, K in ((16, 16), (272, 400), (1408, 2048), (128, 4096))]):
            assert p["wide"] == 0, counts
    for counts in EXPERTS_MANY:
        for p in plan([(sum(counts) + 6, len(counts), N, K, 148, 1) for N, K in EXPERTS_MANY_LAYERS]):
            assert p["wide"] == 1, counts
    cuts = {p["cut"] for p in plan([(M, 1, N, K, 148, 0) for M, N, K in FEW])}
    assert {1, 2, 4, 5, 8} <= cuts, cuts
