"""How cross attention is cut into launches: the host's own rules (csrc/ts3_cross_rules.h), compiled here, on 256
compute units."""
import json
import os
import random
import shutil
import subprocess

import pytest

from cross_shapes import FEW_PARTS, LDS_ROWS, LDS_STATES, MANY, WHOLE

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <hip/hip_runtime.h>
#include <cstdio>
#include "ts3_cross_rules.h"
using namespace ts3;
template <int P, int DP> void plan(const CrossSize &c, int64_t cus) {
    const CrossPlan f = cross_forward_plan<P, DP>(c, cus);
    const CrossBackwardPlan b = cross_backward_plan<P, DP>(c, cus);
    constexpr int DQW = CROSS_DQ_WAVES<DP * P>;
    const long long fw = f.kind == CROSS_ONE ? 1 : f.kind == CROSS_FOUR ? 4 : 16, bw = b.kind == CROSS_ALL ? DQW : 4;
    printf("{\"DP\": %d, \"fits\": %s, \"kind\": %d, \"blocks\": %lld, \"splits\": %lld, \"per\": %lld, \"join\": %d, \"waves\": %lld, "
           "\"dq_kind\": %d, \"qblocks\": %lld, \"qsplits\": %lld, \"dq_waves\": %lld, \"vblocks\": %lld, \"vsplits\": %lld, \"vper\": %lld}\n",
           DP, cross_fits(c) ? "true" : "false", f.kind, (long long)f.blocks, (long long)f.cut.splits, (long long)f.cut.per, f.join, fw,
           b.kind, (long long)b.qblocks, (long long)b.q.splits, bw, (long long)b.vblocks, (long long)b.v.splits, (long long)b.v.per);
}
template <int P> void widths(int D, const CrossSize &c, int64_t cus) {
    if (D <= 16) plan<P, 16>(c, cus);
    else if (D <= 32) plan<P, 32>(c, cus);
    else if (D <= 64) plan<P, 64>(c, cus);
    else plan<P, 128>(c, cus);
}
int main() {
    long long P, D, B, HK, R, S, lengths;
    while (scanf("%lld %lld %lld %lld %lld %lld %lld", &P, &D, &B, &HK, &R, &S, &lengths) == 7) {
        const CrossSize c{B, HK, R, S, lengths != 0};
        if (P == 1) widths<1>((int)D, c, 256);
        else widths<3>((int)D, c, 256);
    }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """plans([(dtype, B, N, S, H, HK, D, lengths), ..]): how each is cut."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.hip").write_text(PROGRAM)
    r = subprocess.run([hipcc, "--cuda-host-only", "--offload-arch=gfx950", "-std=c++17",
                        "-I" + os.path.join(ROOT, "paper_2602_04940_amd", "csrc"), "-o", str(d / "rules"), str(d / "rules.hip")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def run(cases):
        lines = [f"{1 if dtype == 'bf16' else 3} {D} {B} {HK} {N * (H // HK)} {S} {int(lengths)}"
                 for dtype, B, N, S, H, HK, D, lengths in cases]
        out = subprocess.run([str(d / "rules")], input="\n".join(lines), capture_output=True, text=True, check=True)
        res = [json.loads(l) for l in out.stdout.splitlines()]
        assert len(res) == len(cases)
        return res
    return run


ONE, FOUR, ALL = 0, 1, 2
WHOLE_ROWS, JOIN_FEW, JOIN = 0, 1, 2


def test_meshes_of_hundreds_of_millions_of_points_are_accepted(plans):
    def fits(*c):
        return plans([("bf16", *c, False)])[0]["fits"]
    assert fits(1, 100_000_000, 512, 8, 8, 16) and fits(1, 268_435_000, 64, 8, 8, 32) and fits(1, 100_000_000, 64, 8, 1, 16)
    assert fits(1, 8, 268_435_000, 8, 8, 32) and fits((1 << 24) - 1, 1, 128, 1, 1, 16)
    assert not fits(1, 1 << 28, 64, 8, 8, 32) and not fits(1, 8, 1 << 28, 8, 8, 32) and not fits(1 << 24, 1, 1, 1, 1, 16)
    assert not fits(1, (1 << 31) - 1023, 1, 1, 1, 16) and not fits(1, 1, (1 << 31) - 1023, 1, 1, 16)


def _sizes():
    """From one sample to as many as are accepted, and from one row to many."""
    rng = random.Random(1)
    for dtype in ("bf16", "fp32"):
        for D in (16, 32, 64, 128):
            for lengths in (False, True):
                for B, N, S, H in ((1, 1, 1, 1), (5_700_000, 1, 1, 1), (1 << 22, 33, 16, 1), (1 << 19, 64, 64, 8), (2048, 64, 512, 8),
                                   (16, 33, 512, 16), (129, 4000, 300, 1), (257, 1 << 15, 100, 1), (1, 100_000_000, 512, 1)):
                    yield dtype, B, N, S, H, H, D, lengths
                for _ in range(300):
                    HK, G = 2 ** rng.randint(0, 6), 2 ** rng.randint(0, 3)
                    yield (dtype, int(2 ** rng.uniform(0, 24)), int(2 ** rng.uniform(0, 27)), int(2 ** rng.uniform(0, 20)), HK * G, HK, D, lengths)


def test_grids_hold_fewer_than_2_32_threads(plans):
    cases = list(_sizes())
    seen = 0
    for c, p in zip(cases, plans(cases)):
        if not p["fits"]:
            continue
        seen += 1
        pairs = c[1] * c[5]
        for wgs, waves in ((p["blocks"] * p["splits"], p["waves"]), (p["qblocks"] * p["qsplits"], p["dq_waves"]),
                           (p["vblocks"] * p["vsplits"], 4)):
            assert pairs * wgs * waves * 64 < 1 << 32, (c, p)
    assert seen > len(cases) // 3


def test_all_states_in_lds_only_for_workgroups_with_work(plans):
    """Four blocks of 32 rows a wave at least, of the one sample and shared head that a workgroup has."""
    cases = list(_sizes())
    seen = set()
    for c, p in zip(cases, plans(cases)):
        blocks = -(-c[2] * (c[4] // c[5]) // 32)
        for kind, per, waves in ((p["kind"], p["blocks"], p["waves"]), (p["dq_kind"], p["qblocks"], p["dq_waves"])):
            if p["fits"] and kind == ALL:
                seen.add((c[0], c[6], waves))
                assert blocks >= 4 * waves * per, (c, p)
    assert {("bf16", 16), ("bf16", 32), ("bf16", 64), ("fp32", 16)} == {s[:2] for s in seen}


def test_all_states_in_lds_only_where_the_compute_units_have_work(plans):
    """Of the rounds of workgroups, each alone on its unit, seven tenths at least."""
    cases = [("bf16", pairs, 1 << 15, 300, 1, 1, 32, False) for pairs in range(1, 1100)]
    taken = 0
    for c, p in zip(cases, plans(cases)):
        for kind, per in ((p["kind"], p["blocks"]), (p["dq_kind"], p["qblocks"])):
            if kind == ALL:
                taken += 1
                assert c[1] * per >= 0.7 * 256 * -(-c[1] * per // 256), (c, p)
    assert taken > 1100


@pytest.mark.parametrize("lengths", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_shapes_reach_what_they_are_for(plans, dtype, lengths):
    few = plans([(dtype, *c, lengths) for c in FEW_PARTS])
    assert all(p["kind"] == FOUR and p["join"] == JOIN_FEW and p["splits"] > 1 for p in few)
    assert {p["DP"] for p in few} == {16, 32, 64, 128} and max(p["splits"] for p in few) >= 12
    whole = [c for c in WHOLE if dtype == "bf16" or c[5] == 16]
    assert all(p["kind"] == p["dq_kind"] == ALL for p in plans([(dtype, *c, lengths) for c in whole]))
    kinds = [p["kind"] for p in plans([(dtype, *c, lengths) for c in MANY])]
    assert kinds == [FOUR, ONE, FOUR, ALL if dtype == "bf16" else FOUR, ALL]
    B, N, H, HK = LDS_ROWS
    for (t, D), S in LDS_STATES.items():
        if t == dtype:
            last, first = plans([(dtype, B, N, s, H, HK, D, lengths) for s in (S, S + 1)])
            assert last["kind"] == last["dq_kind"] == ALL and first["kind"] == first["dq_kind"] == FOUR


def test_shapes_of_the_first_tests_reach_the_other_kernels(plans):
    """A wave alone, with parts joined by a workgroup; four waves, whole and in parts; dq in parts; dk and dv in parts."""
    from test_gpu_conditioned import CROSS
    for dtype in ("bf16", "fp32"):
        got = plans([(dtype, *c, False) for c in CROSS])
        assert {(p["kind"], p["join"]) for p in got} >= {(ONE, JOIN), (ONE, WHOLE_ROWS), (FOUR, WHOLE_ROWS), (FOUR, JOIN)}
        assert {p["qsplits"] > 1 for p in got} == {p["vsplits"] > 1 for p in got} == {False, True}
