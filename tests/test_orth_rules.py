"""Which products of orthogonalised updates the GPU tests reach: the host's own rule (csrc/ts3_orth_rules.h), compiled
here, on 256 compute units.  A rule that changes may not drop a kernel from the tests unnoticed."""
import math
import os
import shutil
import subprocess

import pytest

from orth_shapes import REACHED, STREAM

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <hip/hip_runtime.h>
#include <cstdio>
#include <vector>
#include "ts3_orth_rules.h"
using namespace ts3;
int main() {
    int lists;
    if (scanf("%d", &lists) != 1) return 1;
    for (int i = 0; i < lists; ++i) {
        int count;
        if (scanf("%d", &count) != 1) return 1;
        std::vector<OrthEntry> e(count);
        for (OrthEntry &m : e)
            if (scanf("%d %d %d", &m.r, &m.c, &m.nb) != 3) return 1;
        for (bool update : {false, true}) {
            const OrthShape s = orth_shape(e.data(), e.size(), update, 256);
            int64_t tiles = 0;
            for (const OrthEntry &m : e) tiles += orth_tiles(m, s.side, update);
            printf("%d %d %lld ", s.side, s.groups, (long long)tiles);
        }
        printf("\n");
    }
}
"""


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    """shapes(lists): ((side, groups, tiles) of the symmetric products, those of the update) of each."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.hip").write_text(PROGRAM)
    r = subprocess.run([hipcc, "--cuda-host-only", "--offload-arch=gfx950", "-std=c++17",
                        "-I" + os.path.join(ROOT, "paper_2602_04940_amd", "csrc"), "-o", str(d / "rules"), str(d / "rules.hip")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def run(lists):
        words = [str(len(lists))]
        for l in lists:
            words.append(str(len(l)))
            words += [f"{min(s[-2:])} {max(s[-2:])} {math.prod(s[:-2])}" for s in l]
        out = subprocess.run([str(d / "rules")], input=" ".join(words), capture_output=True, text=True, check=True)
        rows = [[int(v) for v in l.split()] for l in out.stdout.splitlines()]
        return [(tuple(r[:3]), tuple(r[3:])) for r in rows]
    return run


def test_lists_reach_the_tiles_of_128(shapes):
    got = shapes(STREAM)
    assert [tuple(s[0] == 128 for s in l) for l in got] == REACHED
    for kind in (0, 1):  # one tile a workgroup, and several, whose copies go on across a tile's end
        tiles = [l[kind][2] for l in got if l[kind][0] == 128]
        assert any(t <= 256 for t in tiles) and any(t > 4 * 256 for t in tiles)


def test_other_lists_reach_the_tiles_of_64(shapes):
    from test_gpu_conditioned import ORTH
    got = shapes([l for l in ORTH if any(max(s[-2:]) > 64 for s in l)])
    for kind in (0, 1):
        assert {l[kind][:2] for l in got} >= {(64, 1), (64, 4)}
