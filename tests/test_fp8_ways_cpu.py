"""Which kernel of the 8-bit product takes which sizes, on the CPU: the header that says so, compiled by the host compiler.  The sizes that
tests/test_gpu_fp8_forms.py runs reach every kernel that is built, each with enough blocks to go several times round its place in LDS."""
import os
import subprocess

import pytest

import test_gpu_fp8_forms as forms

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_14272_amd", "csrc")

HARNESS = r"""
#include <cstdio>
#include "fp8_ways.h"
using namespace crisp;
static int blocks(long n) { return (int)((n + 127) / 128); }
int main() {
    char what;
    long T, S, K;
    while (scanf(" %c %ld %ld %ld", &what, &T, &S, &K) == 4) {
        if (what == 'g') {
            const Fp8Size a = {(int)T, (int)K, blocks(S), true, true}, b = {(int)S, (int)K, blocks(T), false, false};
            const bool split = fp8_takes_split(a, a.kb * 128) || fp8_takes_split(b, b.kb * 128);
            printf("pair%d\n", split ? 0 : fp8_pairs(a, b));
            continue;
        }
        for (int v = 0; v < 4; ++v) {           // fp32 and bf16 results, a scale for 128 x 128 of W or for each of its rows
            const Fp8Size z = {(int)T, (int)S, blocks(K), v >= 2, v % 2 == 0};
            if (what == 'r') printf("%s%d ", fp8_takes_raw(T, z.kb) ? "raw" : "none", fp8_split_waves(z.kb));
            else if (fp8_takes_split(z, z.kb * 128)) printf("split%d-%d ", fp8_split_estimate(z, 2) < fp8_split_estimate(z, 1) ? 2 : 1, fp8_split_waves(z.kb));
            else printf("tile%d ", fp8_tile_shape(z));
        }
        printf("\n");
    }
}
"""

TYPES = ("fp32 tiles", "fp32 rows", "bf16 tiles", "bf16 rows")
# blocks that are more than three times round a kernel's place for them (and leave a ragged last round): stages, times the groups that take
# them in turn; two for each of the waves without staging
LEAST = {"tile0": 21, "tile1": 4, "tile2": 7, "tile3": 21, "tile4": 7, "tile5": 13, "tile6": 7, "tile7": 10, "tile8": 7, "tile9": 7,
         "split1-8": 31, "split2-8": 31, "split1-16": 65, "split2-16": 65, "raw8": 9, "raw16": 33}
# shapes of tiles that are built for some types only
ONLY = {"tile3": TYPES[2:], "tile4": TYPES[:2], "tile5": TYPES[2:3], "tile7": TYPES[2:], "tile8": TYPES[2:], "tile9": TYPES[2:3]}


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("fp8_ways") / "ways")
    r = subprocess.run(["g++", "-std=c++17", "-Wall", "-Wno-unused-const-variable", "-ffp-contract=off", "-I", CSRC, "-x", "c++", "-", "-o", exe],
                       input=HARNESS, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(what, sizes):
        lines = "".join("%s %d %d %d\n" % (what, *s) for s in sizes)
        out = subprocess.run([exe], input=lines, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(sizes)
        return [l.split() for l in out]
    return run


def test_sizes_reach_every_kernel(ways):
    seen = set()
    for what, sizes in (("p", forms.LONG), ("r", forms.RAW)):
        for (T, S, K), row in zip(sizes, ways(what, sizes)):
            for way, kind in zip(row, TYPES):
                if -(-K // 128) >= LEAST[way]:
                    seen.add((way, kind))
    built = {(way, kind) for way in LEAST for kind in ONLY.get(way, TYPES)}
    assert seen == built, sorted(built ^ seen)


def test_gradients_reach_one_launch_and_two(ways):
    assert {w[0] for w in ways("g", forms.GRADIENTS)} == {"pair0", "pair1", "pair2"}


def test_few_rows_follow_the_launch_that_quantises(ways):
    """A product that a layer could run in one launch is summed in that launch's order, whatever its other sizes."""
    sizes = [(T, S, K) for T in (1, 2, 7, 16) for S in (1, 100, 4096, 60000) for K in (1, 128, 1024, 128 // T * 128)]
    for (T, S, K), raw, way in zip(sizes, ways("r", sizes), ways("p", sizes)):
        assert T * -(-K // 128) <= 128 and all(w.startswith("raw") for w in raw) and all(w.startswith("split") for w in way)
    sizes = [(17, 100, 128), (16, 100, 1025), (1, 100, 128 * 128 + 1)]
    assert all(w.startswith("none") for row in ways("r", sizes) for w in row)
