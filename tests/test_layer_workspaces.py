"""A workspace made for the largest minibatch serves all smaller ones: sizes do not shrink as rows grow, and each call's own need is within them.
The plans are plain C++ (layer_internal.h), compiled here into a small host program; no GPU is touched."""
import os
import subprocess

import numpy as np
import pytest

from paper_1512_02595_amd import layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include "layer_internal.h"
// For each H, A, last, step read: rows from 1 to `last`; the numbers of those for which a plan needs more than they, or fewer rows before them, were
// told, of those for which less was told than before, of those whose plan needs less than one before, and the bytes told and needed for the last.
int main()
{
    int H, A, last, step;
    while (std::scanf("%d %d %d %d", &H, &A, &last, &step) == 4) {
        size_t told = 0, needed = 0, most = 0;
        int short_of = 0, shrunk = 0, less = 0;
        for (int rows = 1; rows <= last; rows += step) {
            const size_t t = layer::gradient_bytes(rows, H, A);
            needed = layer::gradient_plan(rows, H, A).bytes;
            less += needed < most;
            most = needed > most ? needed : most;
            short_of += t < most;
            shrunk += t < told;
            told = t;
        }
        std::printf("%d %d %d %zu %zu %zu\n", short_of, shrunk, less, told, needed, most);
    }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("layer_plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_1512_02595_amd", "csrc"),
                    str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)

    def ask(H, A, last, step):
        out = subprocess.run([str(d / "plan")], input=f"{H} {A} {last} {step}", capture_output=True, text=True, check=True).stdout
        return tuple(map(int, out.split()))
    return ask


@pytest.mark.parametrize("H, A", [(2048, 29), (2048, 61), (2048, 172), (2048, 1000), (2048, 6000), (1111, 4733), (200, 300), (64, 29), (512, 64),
                                  (513, 65), (768, 2000), (4096, 8000), (16384, 20), (16384, 1 << 20), (1, 1), (1, 1 << 20), (129, 127)])
def test_every_plan_fits_what_was_told_for_more_rows(plans, H, A):
    short_of, shrunk, less, told, needed, most = plans(H, A, 60000, 31)
    assert short_of == 0 and shrunk == 0
    print(H, A, less, told, needed, most)
    assert told <= 7 * most                              # (6.3 times the most that a plan needed, at worst, and once in a hundred sizes)


def test_sizes_of_all_kinds(plans):
    rng = np.random.default_rng(1)
    for H, A, last in zip(*(np.exp(rng.uniform(0, np.log(top), 60)).astype(int) for top in (16385, 20000, 400000))):
        short_of, shrunk, *_ = plans(H, A, last, max(1, last // 500))
        assert short_of == 0 and shrunk == 0, (H, A, last)


def test_some_plans_need_less_for_more_rows(plans):
    """What the sizes have to make up for: where slabs, or the kind of tile, change."""
    assert plans(2048, 6000, 9000, 32)[2] and plans(2048, 172, 33000, 32)[2] and plans(2048, 29, 9000, 32)[2]


@pytest.mark.parametrize("H, A", [(2048, 29), (2048, 172), (2048, 6000), (768, 2000)])
def test_the_librarys_sizes_do_not_shrink(H, A):
    for size in (lambda rows: layer.weight_gradient_workspace_size(rows, H, A), lambda rows: layer.rms_norm_workspace_size(rows, H)):
        told = [size(rows) for rows in [*range(1, 300, 7), *range(300, 36000, 288), 1 << 20, 1 << 30]]
        assert told == sorted(told) and all(n % 256 == 0 for n in told)
