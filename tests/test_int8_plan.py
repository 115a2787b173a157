"""Which tiles a product of the 8-bit layer takes, and the numbering of its tiles (csrc/svdq_int8_plan.h, host code)."""
import subprocess

import pytest

from paper_2605_27003_amd.build import CSRC, HIPCC

DRIVER = """
#include <cstdio>
#include <cstdlib>
#include "svdq_int8_plan.h"
using namespace svdq;
int main(int n, char** v) {
    for (int i = 1; i + 4 < n; i += 5) {
        const Int8Plan p = int8_plan(atol(v[i]), atoi(v[i + 1]), atoi(v[i + 2]), atoi(v[i + 3]), atoi(v[i + 4]) != 0);
        const Int8TileShape s = int8_tile_shape(p.tiles);
        printf("%d %d %d %d\\n", p.cost >= 0.0, s.bm, s.bn, s.stage == 0.0);
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.hip").write_text(DRIVER)
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I", CSRC, str(d / "plan.hip"), "-o", str(d / "plan")], check=True, capture_output=True)

    def ask(*calls):
        out = subprocess.run([str(d / "plan"), *(str(v) for c in calls for v in c)], check=True, capture_output=True, text=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def test_every_call_has_tiles_that_can_be_numbered(plan):
    calls = [(M, N, K, E, f32) for M in (1, 15, 16, 17, 100, 1000, 32760, 75600, 1 << 26) for N in (1, 10, 100, 5120, 30720) for K in (16, 128, 5120, 32768)
             for E in (0, 1, 7, 1024) for f32 in (0, 1)]
    for (M, N, K, E, _), (ok, bm, bn, few) in zip(calls, plan(*calls)):
        assert ok == 1
        row_tiles = M // bm + min(M, E) if E else -(-M // bm)
        assert row_tiles * -(-N // bn) + 256 < 1 << 31
    # what no tile can number is refused, not cut short
    assert plan((1 << 26, 1 << 30, 64, 0, 0))[0][0] == 0


def test_few_tokens_and_many(plan):
    """Single tokens take the kernel that splits K; what fills the chip several times over the largest tiles; both from either form."""
    (one, many, decode, prompt) = plan((1, 5120, 5120, 0, 0), (32760, 5120, 5120, 0, 0), (32, 2816, 2048, 64, 0), (32760, 5120, 5120, 2, 0))
    assert one[3] == 1 and decode[3] == 1 and many[1:3] == (256, 256) and prompt[1:3] == (256, 256)
