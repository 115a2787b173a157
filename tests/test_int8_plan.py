"""Which tiles a product of the 8-bit layer takes, and the numbering of its tiles (csrc/svdq_int8_plan.h, host code)."""
import subprocess

import pytest

from paper_2605_27003_amd.build import CSRC, HIPCC
from tests.int8_products import PRODUCTS

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


KERNELS = """
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>
#include <string>
#include "svdq_int8_plan.h"
using namespace svdq;
static const char* kernel(long M, int N, int K, int E, bool f32) {
    static char text[100];
    const Int8Kernel k = int8_kernel(int8_plan(M, N, K, E, f32).tiles, M, N, K, E);
    const Int8TileShape s = int8_tile_shape(k.tiles);
    sprintf(text, "%d %d %d %d", s.bm, s.bn, k.depth, k.lines);
    return text;
}
int main(int n, char** v) {
    for (int i = 1; i + 3 < n; i += 4)
        for (int f32 = 0; f32 < 2; ++f32) puts(kernel(atol(v[i]), atoi(v[i + 1]), atoi(v[i + 2]), atoi(v[i + 3]), f32));
    if (n > 1) return 0;
    // any call: sizes even on their logarithms, half of the K of whole stages, half not grouped
    std::mt19937_64 random(1);
    auto size = [&](double low, double high) { return std::exp(std::uniform_real_distribution<double>(std::log(low), std::log(high + 1))(random)); };
    std::set<std::string> seen;
    for (int i = 0; i < 400000; ++i) {
        const int E = random() % 2 ? (int)size(1, 1024) : 0, N = (int)size(1, 40000), k16 = (int)size(1, 2048), K = random() % 2 ? 16 * k16 : (16 * k16 + 127) / 128 * 128;
        const long M = (long)size(1, 100000);
        for (int f32 = 0; f32 < 2; ++f32) {
            char of[32];
            sprintf(of, " %d %d %d", K % 128 == 0, E > 0, f32);
            seen.insert(kernel(M, N, K, E, f32) + std::string(of));
        }
    }
    for (auto& s : seen) puts(s.c_str());
}
"""


def test_products_of_the_gpu_tests_reach_every_kernel(tmp_path):
    """Each takes the kernel that it is listed under; and no call takes a kernel, in its forms for K of whole stages or not, grouped or not, bf16 or binary32,
    that none of them takes."""
    (tmp_path / "kernels.hip").write_text(KERNELS)
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I", CSRC, str(tmp_path / "kernels.hip"), "-o", str(tmp_path / "kernels")], check=True, capture_output=True)
    ask = lambda *v: [tuple(map(int, line.split())) for line in subprocess.run([str(tmp_path / "kernels"), *map(str, v)], check=True, capture_output=True, text=True).stdout.splitlines()]
    calls = [(kernel, call) for kernel, calls in PRODUCTS.items() for call in calls]
    took = ask(*(v for _, call in calls for v in call))
    assert len(took) == 2 * len(calls)
    wrong = [(kernel, call, now) for (kernel, call), now in zip(calls, took[::2]) if now != tuple(map(int, kernel))]
    assert not wrong, wrong
    tested = {(*now, int(call[2] % 128 == 0), int(call[3] > 0), f32) for f32 in (0, 1) for (_, call), now in zip(calls, took[f32::2])}
    taken = set(ask())
    assert len(taken) >= 90 and not taken - tested, taken - tested
