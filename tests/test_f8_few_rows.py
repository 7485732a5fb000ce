"""Few rows of A: the plan takes the form that was measured to be the faster one, where the two were clearly apart."""
import os
import subprocess

import paper_2508_03984_amd as oz

PLAN = r"""
#include "%s"
#include <cstdio>
using namespace oz2;
int main() {
    long m, n, k; int gated;
    while (scanf("%%ld %%ld %%ld %%d", &m, &n, &k, &gated) == 4) printf("%%d\n", (int)f8_plan(m, n, k, gated).form);
}
"""
# (m, n, k, gated): us of the form for few rows | of the best tiles
MEASURED = {
    (1, 8192, 8192, 0): (13.7, 16.2), (8, 8192, 8192, 0): (15.1, 15.6), (17, 8192, 8192, 0): (19.6, 16.0), (64, 8192, 8192, 0): (41.6, 18.1),
    (17, 4096, 4096, 0): (7.4, 9.4), (32, 4096, 4096, 0): (8.7, 9.9), (17, 4096, 16384, 0): (21.0, 16.6), (16, 16384, 4096, 0): (18.0, 13.9),
    (17, 2048, 2048, 0): (4.6, 6.5), (33, 2048, 2048, 0): (6.0, 7.0), (64, 2048, 2048, 0): (7.3, 7.9),
    (20, 4440, 6221, 0): (16.5, 11.9), (24, 5120, 5120, 0): (15.2, 11.4), (40, 5120, 5120, 0): (21.6, 12.2),
    (23, 84, 11286, 0): (15.3, 8.5), (60, 84, 4000, 0): (11.6, 7.2), (16, 1000, 3000, 0): (5.2, 7.7), (24, 1000, 3000, 0): (6.0, 7.8),
    (4, 16384, 4096, 1): (29.2, 32.0), (16, 16384, 4096, 1): (28.9, 34.3), (64, 16384, 4096, 1): (56.5, 33.5),
    (17, 8192, 8192, 1): (31.7, 34.1), (17, 11000, 4096, 1): (22.7, 18.6), (20, 4944, 6158, 1): (22.1, 16.3), (33, 2048, 2048, 1): (7.3, 8.3),
}


def test_the_faster_form(tmp_path):
    (tmp_path / "plan.cpp").write_text(PLAN % os.path.join(os.path.dirname(oz.lib_path()), "csrc", "oz2_f8.hpp"))
    subprocess.check_call(["g++", "-O1", "-std=c++17", str(tmp_path / "plan.cpp"), "-o", str(tmp_path / "plan")])
    out = subprocess.run([str(tmp_path / "plan")], input="\n".join("%d %d %d %d" % c for c in MEASURED), capture_output=True, text=True, check=True).stdout
    slower = [c for c, form in zip(MEASURED, out.split()) if (form == "0") != (MEASURED[c][0] < MEASURED[c][1])]
    assert not slower
