"""Which kernels the shapes of tests/test_gpu_class_tiles.py run, from the rules in csrc/launch_sizes.h: the tiles that the lists name, every one
there is, and at least one whole turn of its ring of stages (no GPU needed)."""
import importlib.util
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_1805_10111_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "launch_sizes.h"
using namespace dq;
static const char *name(TileSize s) { const char *const names[] = {"Large", "Half", "Middle", "Few", "Fewest"}; return names[s]; }
int main()
{
    long n, c, d;
    int parts, four;
    while (std::scanf("%ld %ld %ld %d %d", &n, &c, &d, &parts, &four) == 5) {
        const TileSize s = tile_for_rows(c, n, parts, !four);
        const TileDims t = dims_of(s, parts, false);
        const int64_t piece = piece_of(c, ceil_div(n, t.y) * t.y, planes_of_g(parts, t.x)), split = da_split(n, d, piece, parts);
        std::printf("%s %s %s %ld %ld %ld\n", name(s), name(tile_for_da(n, d)), name(tile_for_dw(n, c, d, piece, parts)), (long)ceil_div(c, piece),
                    (long)ceil_div(piece, split), (long)(split < c ? split : c));
    }
}
"""


@pytest.fixture(scope="module")
def shapes():
    spec = importlib.util.spec_from_file_location("class_tile_shapes", os.path.join(HERE, "test_gpu_class_tiles.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture(scope="module")
def tiles(tmp_path_factory):
    at = tmp_path_factory.mktemp("tiles")
    (at / "tiles.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", CSRC, str(at / "tiles.cpp"), "-o", str(at / "tiles")], check=True)

    def of(cases):
        lines = "".join(f"{n} {c} {d} {int(t == 'f32')} {int(t == 'mx4')}\n" for t, n, c, d in cases)
        out = subprocess.run([str(at / "tiles")], input=lines, capture_output=True, text=True, check=True).stdout.split("\n")
        return [(s, da, dw, int(pieces), int(splits), int(each)) for s, da, dw, pieces, splits, each in (line.split() for line in out if line)]
    return of


def turn(t, tile):
    """Columns, rows or classes that one turn of a tile's ring takes: stages of one step (small tiles of 16 bits: two), four of them, in
    float32's larger tiles two, in half tiles six (where operands are read two by two, in three places)."""
    if t == "f32":
        return 32 * (4 if tile in ("Few", "Fewest") else 2)
    return 32 * (8 if tile in ("Few", "Fewest") else 6 if tile == "Half" else 4)


def test_unit_features(shapes, tiles):
    seen = set()
    for cases, several in ((shapes.UNIT_FEATURES, False), (shapes.SEVERAL_PIECES, True)):
        for (t, n, c, d, scores, dw), (s, _, w, pieces, _, _) in zip(cases, tiles([x[:4] for x in cases])):
            edge = ":edge" if t != "f32" and d % 8 == 0 and d % 32 else ""      # (the tests' rows are 16-byte aligned ones where d allows it)
            assert (s + edge, w, pieces > 1) == (scores, dw, several), (t, n, c, d)
            assert n <= d and d > turn(t, s), (t, n, c, d)
            seen |= {(t, "grad" if several else "scores", scores), (t, "dw", w)}
            if w != "Few" and not several and n > turn(t, w):
                seen.add((t, "dw's ring", w))
    for t in ("bf16", "f16"):
        # (the smaller tiles look for rows' ends in any case: with and without are one kernel)
        for kind, sizes in (("scores", ("Large", "Large:edge", "Half", "Half:edge", "Middle", "Middle:edge", "Few", "Few:edge", "Fewest", "Fewest:edge")),
                            ("dw", ("Half", "Middle", "Few")), ("dw's ring", ("Half", "Middle"))):
            assert {x for x in sizes if (t, kind, x) not in seen} == set(), (t, kind)
    for size in ("Large", "Half", "Few", "Fewest"):
        assert {(t, e) for t in ("bf16", "f16") for e in ("", ":edge") if (t, "grad", size + e) in seen} >= {("bf16", ":edge"), ("f16", "")}
    for kind, sizes in (("scores", ("Large", "Middle", "Few", "Fewest")), ("grad", ("Large", "Few", "Fewest")), ("dw", ("Large", "Middle", "Few")),
                        ("dw's ring", ("Large", "Middle"))):
        assert {x for x in sizes if ("f32", kind, x) not in seen} == set(), kind


def test_unit_classes(shapes, tiles):
    seen = set()
    for (t, n, c, d, da, splits), (_, a, _, pieces, parts, each) in zip(shapes.UNIT_CLASSES, tiles([x[:4] for x in shapes.UNIT_CLASSES])):
        assert (a, "several" if parts > 1 else "one", pieces) == (da, splits, 1), (t, n, c, d)
        seen.add((t, a))
        if each > turn(t, a):
            seen.add((t, a, "ring"))
    assert seen >= {(t, a) for t in ("f32", "f16", "bf16") for a in ("Large", "Middle", "Few", "Fewest")}
    assert {x for x in ((t, a, "ring") for t in ("f32", "f16", "bf16") for a in ("Large", "Middle", "Few", "Fewest")) if x not in seen} == set()


def test_products_in_four_bits(shapes, tiles):
    got = tiles([("mx4", n, c, 128 * g) for n, c, g, _ in shapes.PRODUCTS])
    assert [x[0] for x in got] == [tile for *_, tile in shapes.PRODUCTS]
    assert {x[0] for x in got} == {"Large", "Middle", "Few", "Fewest"}
    for n, c, g, tile in shapes.PRODUCTS:
        if tile != "Large":
            assert g >= (8 if tile in ("Few", "Fewest") else 4)          # stages of two groups or one, four to a turn
