"""The rules by which the output layer's calls take one kernel or another (layer_internal.h), compiled into a small host program."""
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "layer_internal.h"
int main()
{
    char what[16];
    int rows, H, A, list;
    while (std::scanf("%15s %d %d %d %d", what, &rows, &H, &A, &list) == 5) {
        if (!std::strcmp(what, "rows")) {
            const layer::RowShape s = layer::row_shape(rows, H);
            std::printf("%d %d\n", s.waves, s.elements);
        } else if (!std::strcmp(what, "product")) {
            const layer::ProductTile t = layer::product_tile(rows, H, A, list != 0);
            std::printf("%d %d\n", t.rows, t.symbols);
        } else {
            const layer::GradientPlan p = layer::gradient_plan(rows, H, A);
            std::printf("%d %d\n", p.symbols, p.slabs);
        }
    }
}
"""


@functools.lru_cache(None)
def _ask(question):
    if not hasattr(_ask, "program"):
        _ask.folder = tempfile.TemporaryDirectory()
        source, _ask.program = os.path.join(_ask.folder.name, "rules.cpp"), os.path.join(_ask.folder.name, "rules")
        with open(source, "w") as f:
            f.write(PROGRAM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_1512_02595_amd", "csrc"),
                        source, "-o", _ask.program], check=True)
    return tuple(map(int, subprocess.run([_ask.program], input=question, capture_output=True, text=True, check=True).stdout.split()))


def row_shape(rows, H):
    """(wavefronts to a row, elements to a lane) for rows to 8 bits and the norm."""
    return _ask(f"rows {rows} {H} 1 0")


def product_tile(rows, H, A, listed):
    """(rows, symbols) of a workgroup's tile."""
    return _ask(f"product {rows} {H} {A} {int(listed)}")


def gradient_tile(rows, H, A):
    """(symbols of a tile, slabs of rows)."""
    return _ask(f"gradient {rows} {H} {A} 0")
