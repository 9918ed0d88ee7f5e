"""Which loops and pipelines of the gated feed-forward's kernels the GPU tests reach: the host's own
rules (csrc/ts3_gated_rules.h), compiled here, cut the tests' sizes on 256 compute units, and every
kernel has to run long enough for its slots and registers to be used again.  A rule that changes
may not drop a loop from the tests unnoticed."""
import json
import os
import shutil
import subprocess

import pytest

from gated_shapes import LONG, MIDDLE

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <hip/hip_runtime.h>
#include <cstdio>
#include <cstdlib>
#include "ts3_gated_rules.h"
using namespace ts3;
template <int P, int CP> void plan(int64_t N, int F, int64_t tile, int cus) {
    const int chunks = (F + 31) / 32;
    constexpr int PTS = GatedShape<P, CP>::PTS;
    constexpr bool WIDE = GatedWide<P, CP>::USE;
    constexpr int PTX = WIDE ? GatedWide<P, CP>::PTS : GatedShapeX<P, CP>::PTS;
    const int64_t nb = (N + PTS - 1) / PTS;
    const int S = gated_splits(N, nb, chunks, P, CP, cus), per = (chunks + S - 1) / S;
    printf("{\"P\": %d, \"CP\": %d, \"chunks\": %d, \"S\": %d, \"per\": %d, \"halves\": %d", P, CP, chunks, S, per,
           gated_halves<P, CP>(nb * S, per, cus));
    printf(", \"wide\": %s, \"ring\": %s, \"waves\": %d, \"slots\": %d, \"tiles\": [", WIDE ? "true" : "false",
           !WIDE && GatedShapeX<P, CP>::RING ? "true" : "false", gated_dw_waves<P, CP>(chunks),
           P == 3 ? 2 : gated_dw_waves<P, CP>(chunks) == 8 ? GatedDw<P, CP, 8 * GatedDwWide<P, CP>::USE8 + 4 * !GatedDwWide<P, CP>::USE8>::SLOTS
                                                          : GatedDw<P, CP, 4>::SLOTS);
    const int64_t step = tile < N ? tile : N;
    const int SP = gated_point_splits<P, CP>(chunks, step, cus);
    for (int64_t t0 = 0; t0 < N; t0 += step) {
        const int64_t m = step < N - t0 ? step : N - t0, tb = (m + PTX - 1) / PTX, tp = tb * PTX;
        const int s = gated_splits(m, tb, chunks, P, CP, cus);
        printf("%s{\"points\": %lld, \"S\": %d, \"per\": %d, \"steps\": %lld}", t0 ? ", " : "", (long long)m, s, (chunks + s - 1) / s,
               (long long)(((tp + SP - 1) / SP + 31) / 32 * 32 / GatedDw<P, CP, 4>::KP));
    }
    printf("]}\n");
}
template <int P> void widths(int C, int64_t N, int F, int64_t tile, int cus) {
    if (C <= 64) plan<P, 64>(N, F, tile, cus);
    else if (C <= 128) plan<P, 128>(N, F, tile, cus);
    else if (C <= 192) plan<P, 192>(N, F, tile, cus);
    else plan<P, 256>(N, F, tile, cus);
}
int main(int argc, char **argv) {
    for (int i = 1; i + 3 < argc; i += 4)
        for (int P : {1, 3}) {
            const int64_t N = atoll(argv[i]), tile = atoll(argv[i + 3]);
            if (P == 1) widths<1>(atoi(argv[i + 1]), N, atoi(argv[i + 2]), tile, 256);
            else widths<3>(atoi(argv[i + 1]), N, atoi(argv[i + 2]), tile, 256);
        }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """{"long": ..., "middle": ...}: the plans of the sizes in both types."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.hip").write_text(PROGRAM)
    r = subprocess.run([hipcc, "--cuda-host-only", "--offload-arch=gfx950", "-std=c++17",
                        "-I" + os.path.join(ROOT, "paper_2602_04940_amd", "csrc"), "-o", str(d / "rules"), str(d / "rules.hip")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def run(shapes):
        out = subprocess.run([str(d / "rules"), *(str(v) for s in shapes for v in s)], capture_output=True, text=True, check=True)
        return [json.loads(l) for l in out.stdout.splitlines()]
    return {"long": run(LONG), "middle": run([(N, C, F, N) for N, C, F in MIDDLE])}


WIDTHS = (64, 128, 192, 256)


@pytest.mark.parametrize("P", [1, 3])
@pytest.mark.parametrize("CP", WIDTHS)
def test_forward_loops(plans, P, CP):
    mine = [p for p in plans["long"] + plans["middle"] if (p["P"], p["CP"]) == (P, CP)]
    assert any(p["halves"] == 1 and p["S"] == 1 and p["per"] >= 4 for p in mine)
    if P == 1 or CP <= 128:  # two waves per SIMD on the same points: alone and in splits, halves alike and not
        alone = [p for p in mine if p["halves"] == 2 and p["S"] == 1]
        assert any(p["per"] == 4 for p in alone) and any(p["per"] == 5 for p in alone)
    assert any(p["S"] > 1 and p["per"] >= 3 for p in mine)


@pytest.mark.parametrize("P", [1, 3])
@pytest.mark.parametrize("CP", WIDTHS)
def test_backward_loops(plans, P, CP):
    """Slopes and dx: at least five chunks per workgroup, in whole blocks and where they are split."""
    tiles = [t for p in plans["long"] if (p["P"], p["CP"]) == (P, CP) for t in p["tiles"]]
    assert any(t["S"] == 1 and t["per"] >= 5 for t in tiles)
    if CP == 256:
        assert any(t["S"] > 1 and t["per"] >= 3 for t in tiles)


def test_every_kernel_of_the_backward_is_there(plans):
    kinds = {(p["P"], p["CP"]): (p["wide"], p["ring"]) for p in plans["long"]}
    assert kinds == {(1, 64): (False, False), (1, 128): (False, False), (1, 192): (True, False), (1, 256): (True, False),
                     (3, 64): (False, False), (3, 128): (True, False), (3, 192): (False, True), (3, 256): (False, True)}


@pytest.mark.parametrize("P", [1, 3])
def test_rotating_loops_end_everywhere(plans, P):
    """dx from the store turns three sets of registers over, the float32 slopes two: long loops with
    each remainder of steps."""
    chunks = [t["per"] for p in plans["long"] if p["P"] == P and p["wide"] for t in p["tiles"] if t["S"] == 1]
    steps = {c * (1 if P == 1 else 2) for c in chunks}
    assert {s % 3 for s in steps if s >= 6} == {0, 1, 2}
    if P == 3:
        assert {c % 2 for c in chunks if c >= 4} == {0, 1}


@pytest.mark.parametrize("P,CP,waves", [(1, 64, 4), (1, 128, 4), (1, 128, 8), (1, 192, 4), (1, 256, 4), (1, 256, 8), (3, 64, 4),
                                        (3, 128, 4), (3, 192, 4), (3, 256, 4)])
def test_weight_gradient_loops(plans, P, CP, waves):
    """Every ring of slots is used at least three times, in a first tile and in one that adds to it."""
    mine = [p for p in plans["long"] if (p["P"], p["CP"], p["waves"]) == (P, CP, waves)]
    assert any(all(t["steps"] >= 3 * p["slots"] for t in p["tiles"][:2]) and len(p["tiles"]) >= 2 and
               p["tiles"][1]["points"] == p["tiles"][0]["points"] for p in mine)
