"""Which form the tests' products take: every form and a sliced reduction for either type of result (CPU)."""
import os
import subprocess

import pytest

from fp8_forms import FORMS, NAMES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
#include <stdio.h>
#include <stdlib.h>

#include "fp8_plan.h"

int main(int argc, char **argv)   // M N K type, any number of times
{
    for (int i = 1; i + 3 < argc; i += 4) {
        const Fp8Plan p = fp8_plan_of(atoi(argv[i]), atoi(argv[i + 1]), (atoi(argv[i + 2]) + 127) / 128, atoi(argv[i + 3]));
        printf("%d %d\\n", p.form, p.slices);
    }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_1805_11046_amd", "csrc"),
                           str(at / "plan.cpp"), "-o", str(at / "plan")])

    def of(*cases):
        out = subprocess.check_output([str(at / "plan")] + [str(v) for c in cases for v in c], text=True)
        return [(NAMES[int(f)], int(z)) for f, z in (line.split() for line in out.splitlines())]

    return of


def test_products_of_the_tests_take_the_forms_that_they_are_there_for(plans):
    for M, N, K, bf16, f32 in FORMS:
        assert plans((M, N, K, 1), (M, N, K, 0)) == [bf16, f32], (M, N, K)


def test_every_form_is_taken(plans):
    for at, without in ((3, ()), (4, ("tile 128 deep",))):       # fp32 results have no deep form
        assert {f[at][0] for f in FORMS} == set(NAMES) - set(without)
        assert {f[at][1] for f in FORMS} >= {1, 4, 8, 16}
    assert all(K > 8 * 128 for _, _, K, _, _ in FORMS)


def test_small_products_of_few_rows_to_bf16_are_direct(plans):
    # their sums are fp32; the tiles' are not
    for case in ((1, 100, 300), (16, 48, 640), (64, 70, 130), (1, 4096, 4096), (2, 6122, 421), (58, 318, 418)):
        assert plans(case + (1,))[0][0].startswith("direct"), case


def test_sizes_at_the_limits_have_a_form(plans):
    big = 1 << 22
    for case in ((1, big, 128, 1), (big, 1, 128, 0), (big, 1 << 14, 128, 1), (1 << 14, big, 1 << 23, 0), (1, 1, 1 << 23, 1), (1, 1, 1, 0), (65, big, 1, 1)):
        form, slices = plans(case)[0]
        assert form in NAMES and 1 <= slices <= 16


def test_the_workspace_holds_the_slices_of_either_type(plans):
    from test_abi import _lib_path
    _lib_path()
    import paper_1805_11046_amd as m
    for M, N, K, bf16, f32 in FORMS:
        most = max(bf16[1], f32[1])
        assert m.binding._lib.q8t_fp8_gemm_workspace_size(M, N, K) == (most * M * N * 4 if most > 1 else 0)
