"""That the sizes of the GPU tests of 8-bit floating-point products reach every form of the kernels: the plan is a matter of fitted times, and another
fit must not leave a form untested."""
import os
import subprocess

import pytest

import f8_sizes
import paper_2508_03984_amd as oz

PLAN = r"""
#include "%s"
#include <cstdio>
using namespace oz2;
int main() {
    long m, n, k; int gated;
    while (scanf("%%ld %%ld %%ld %%d", &m, &n, &k, &gated) == 4) {
        const F8Plan p = f8_plan(m, n, k, gated);
        printf("%%d %%d %%d\n", (int)p.form, p.ranges > 1, f8_items(p.form, m, n, gated) * p.ranges <= 512);
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PLAN % os.path.join(os.path.dirname(oz.lib_path()), "csrc", "oz2_f8.hpp"))
    subprocess.check_call(["g++", "-O1", "-std=c++17", str(d / "plan.cpp"), "-o", str(d / "plan")])

    def forms(sizes, gated):
        text = "\n".join("%d %d %d %d" % (*s, gated) for s in sizes)
        out = subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True).stdout.split()
        return [(int(out[i]), out[i + 1] == "1", out[i + 2] == "1") for i in range(0, len(out), 3)]
    return forms


@pytest.mark.parametrize("gated", [False, True])
def test_sizes_take_the_forms_that_they_stand_for(plan, gated):
    by_form = f8_sizes.GATED if gated else f8_sizes.PRODUCTS
    assert set(by_form) == {(0, False), (1, False), (1, True), (2, False), (2, True), (3, False), (3, True)}
    for form, sizes in by_form.items():
        assert [f[:2] for f in plan(sizes, gated)] == [form] * len(sizes), (form, sizes)
    # tiles of 64 x 64 with two stages and with four
    assert {deep for _, _, deep in plan(by_form[f8_sizes.SMALL, False], gated)} == {False, True}
