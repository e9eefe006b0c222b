"""The second launch choice of the gradients on block-scaled numbers (narrow_plan of csrc/tern_mx_choice.h, host code) over the
sizes that it is asked about: every step of k is somebody's, no share is empty, the workspace is what the shares write, and
a side is only called narrow where csrc/tern_mx_narrow.hip has a kernel for it."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1801_09449_amd", "csrc")

SOURCE = r"""
#include "tern_mx_choice.h"
#include <cstdio>
#include <random>
using namespace tern;

int main()
{
    long lost = 0, empty = 0, many = 0, space = 0, side = 0, unlike = 0, refused = 0, seen[5] = {}, split = 0;
    std::mt19937_64 r(8);
    auto size = [&](int bits) { return 1 + (int64_t)(r() % ((uint64_t)1 << (1 + r() % bits))); };
    for (int i = 0; i < 300000; ++i) {
        const bool input = r() % 2;
        const int64_t parts = 1 + (int64_t)(r() % 3);
        const ProductSize s = {size(r() % 2 ? 7 : 20), size(r() % 2 ? 7 : 20), size(18), parts};
        const int form = r() % 4 ? -1 : (int)(r() % (kForms + 1)), splits = r() % 4 ? 0 : 1 + (int)(r() % kMostSplits);
        ProductPlan p = {-7, -7, -7, -7}, again;
        const bool is = narrow_plan(s, input, form, splits, &p);
        unlike += narrow_plan(s, input, form, splits, &again) != is;
        const bool a_narrow = s.na <= (parts > 1 ? kNarrowInputs : kNarrowRows), any = a_narrow || s.nb <= kNarrowRows;
        if (!is) {
            refused += form == kNarrow && any;              // asked for, and there is a kernel
            refused += p.form != -7;                        // the plan of another kernel is left alone
            continue;
        }
        side += !any || (form >= 0 && form != kNarrow) || p.form != kNarrow;
        side += p.wide != (a_narrow ? (input ? kWideDyRows : kWideDyDown) : input ? kWideWeights : kWideInput);
        // blocks of 32 of the narrow side that the kernels are built for: four where dy is wide and in parts, else two
        const int64_t blocks = ceil_div(a_narrow ? s.na : s.nb, 32);
        side += blocks > (a_narrow && parts > 1 ? 4 : 2);
        const int64_t each = ceil_div(s.groups, p.splits);  // (split_steps of the launch)
        lost += p.splits < 1 || each * p.splits < s.groups || steps_of(kNarrow, s) != s.groups;
        empty += each * (p.splits - 1) >= s.groups;
        many += p.splits > kMostSplits || (splits && p.splits > splits);
        space += p.partial_bytes != (p.splits > 1 ? p.splits * s.nb * ((s.na + 3) / 4 * 4) * 4 : 0);
        unlike += again.splits != p.splits || again.wide != p.wide || again.partial_bytes != p.partial_bytes;
        ++seen[p.wide];
        split += p.splits > 1;
    }
    for (int w = kWideDyRows; w <= kWideInput; ++w) lost += seen[w] < 100;
    std::printf("%ld %ld %ld %ld %ld %ld %ld %d\n", lost, empty, many, space, side, unlike, refused, split > 1000);
}
"""


def test_every_narrow_choice_covers_its_product(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    src = tmp_path / "choice.cpp"
    src.write_text(SOURCE)
    exe = tmp_path / "choice"
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    out = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    assert out == ["0"] * 7 + ["1"]
