"""The rules of 8-bit products and of symmetric products (csrc/launch_sizes.h), without a GPU: the sizes of test_gpu_eight_bit_tiles.py take the kernels that
they are named after, and no symmetric product of two matrices of `side` rows is planned in splits of small tiles, which have no kernel."""
import subprocess

from test_eight_bit_plans import CSRC, HERE, module

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "launch_sizes.h"
using namespace dq;
int main()
{
    // factors along k and across it (two small matrices), of one part or two, alone or two products at a time: whatever the side
    for (long side = 32; side <= 32768; side += 32)
        for (int jobs = 1; jobs <= 2; ++jobs)
            for (int products = 1; products <= 3; products += 2) {
                const GramPlan g = gram_plan(side, side, products, jobs);
                if (g.tiles <= 0 || (g.size == kTileFew && !g.at_once)) { std::printf("FAIL %ld %d %d\n", side, products, jobs); return 1; }
            }
    // one part over any k
    for (long side = 32; side <= 4096; side += 32)
        for (long k = 32; k <= 1 << 20; k += 1 + k / 3) {
            const GramPlan g = gram_plan(side, k, 1, 1);
            if (g.tiles <= 0 || (g.size == kTileFew && !g.at_once)) { std::printf("FAIL %ld over %ld\n", side, k); return 1; }
        }
    long n, c, d;
    while (std::scanf("%ld %ld %ld", &n, &c, &d) == 3)
        for (int f32 = 0; f32 < 2; ++f32) {
            const ProductPlan p = product_plan(n, c, ceil_div(d, 128), f32);
            const long tiles = p.tiles_x * p.tiles_y * p.splits;
            std::printf("%s%s%s %ld\n", p.few ? "strips" : p.size == kTileLarge ? "Large" : "Middle", !p.few && p.size == kTileMiddle ? (tiles <= 256 ? "4" : "2") : "", p.splits > 1 ? "+" : "",
                        static_cast<long>(p.per_split));
        }
    std::printf("swept\n");
}
"""


def test_kernels_of_the_sizes(tmp_path, monkeypatch):
    monkeypatch.syspath_prepend(HERE)
    kinds = module("test_gpu_eight_bit_tiles").KINDS
    (tmp_path / "plans.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", CSRC, str(tmp_path / "plans.cpp"), "-o", str(tmp_path / "plans")], check=True)
    r = subprocess.run([str(tmp_path / "plans")], input="\n".join("%d %d %d" % k for k in kinds.values()), capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-300:]
    lines = r.stdout.split("\n")
    assert lines[2 * len(kinds)] == "swept"
    for i, (kind, (n, c, d)) in enumerate(kinds.items()):
        for line in lines[2 * i:2 * i + 2]:                       # 16-bit results, float32
            name, per = line.split()
            assert name == kind
        blocks = (d + 127) // 128
        assert blocks % 2 == 1 and (int(per) >= blocks if "+" not in kind else blocks % int(per) % 2 == 1)
