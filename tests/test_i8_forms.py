"""Plans of the 8-bit integer products and conversions, on the CPU: that the sizes of the GPU tests reach every form of the kernels (another fit must not leave one
untested), that ranges of k cover it, and that what large tiles leave to smaller ones is what those take."""
import os
import subprocess

import pytest

import paper_2508_03984_amd as oz

PLAN = r"""
#include "%s"
#include <cstdio>
using namespace oz2;
int main() {
    char what; long a, b, c, d;
    while (scanf(" %%c %%ld %%ld %%ld %%ld", &what, &a, &b, &c, &d) == 5) {
        I8Args x{};
        x.groups.offsets = reinterpret_cast<const int32_t *>(&x);
        if (what == 'd') {                                     // m n k
            const I8Plan p = i8_plan(a, b, c);
            x.m = a; x.n = b; x.k = c; x.ranges = p.ranges;
            printf("%%d %%d %%d %%ld %%ld %%u\n", (int)p.form, p.ranges, p.kb_each, (long)p.plane_bytes, (long)i8_tiles(I8Mode::kDense, p.form, x),
                   p.form == I8Form::kLarge && p.ranges == 1 ? i8_left_over(i8_tiles(I8Mode::kDense, p.form, x), 256) : 0);
        } else if (what == 'r' || what == 's') {               // rows groups n k, rows groups m n
            x.groups.rows = a; x.groups.groups = b;
            const I8Mode mode = what == 'r' ? I8Mode::kRows : I8Mode::kSums;
            if (what == 'r') { x.m = a; x.n = c; x.k = d; } else { x.m = c; x.n = d; x.k = a; }
            const I8Plan p = i8_grouped_plan(mode, x);
            x.ranges = p.ranges;
            printf("%%d %%ld %%d %%ld\n", (int)p.form, (long)i8_tiles(mode, p.form, x), p.ranges, (long)p.plane_bytes);
        } else {                                               // rows cols groups, both forms (q: by group, b: a batch)
            I8Quantize q{};
            q.q = q.qt = reinterpret_cast<int8_t *>(&x);
            q.cols = b;
            q.side_by_side = what == 'q';
            q.groups = I8Groups{what == 'q' ? x.groups.offsets : nullptr, (int)c, (int)a, (int)(a / c)};
            const I8ConvertPlan p = i8_convert_plan(q);
            printf("%%d %%d %%d %%d %%ld\n", p.lanes, p.rows_each, p.columns_each, p.strips, (long)i8_quantize_threads(q));
        }
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PLAN % os.path.join(os.path.dirname(oz.lib_path()), "csrc", "oz2_i8.hpp"))
    subprocess.check_call(["g++", "-O1", "-std=c++17", str(d / "plan.cpp"), "-o", str(d / "plan")])

    def ask(what, sizes):
        text = "\n".join("%s %d %d %d %d" % (what, *(list(s) + [0] * 4)[:4]) for s in sizes)
        out = subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        return [tuple(int(v) for v in line.split()) for line in out]
    return ask


def test_sizes_of_the_gpu_tests_take_every_form(plan):
    from test_gpu_i8 import GROUPS, PRODUCTS
    import test_gpu_i8_large as large
    sizes = PRODUCTS + large.PRODUCTS + [(100, 100, 20000), (54, 205, 13245), (3, 16, 40000), (512, 500, 4100), (1300, 1000, 30001)]
    got = plan("d", sizes)
    forms = {(f, r > 1) for f, r, *_ in got}
    assert {(0, False), (1, False), (1, True), (2, False), (3, False), (3, True)} <= forms, forms
    assert any(left for *_, left in got)                      # a last round of large tiles that smaller ones take
    tiles = [t for f, _, _, _, t, _ in got if f == 1]         # with four stages, with three and with two
    assert any(t <= 512 for t in tiles) and any(512 < t <= 768 for t in tiles) and any(t > 768 for t in tiles)
    assert any(m % 256 and n % 256 and k % 128 for (m, n, k), p in zip(sizes, got) if p[0] == 3)
    rows = [(o[-1] + 7, len(o) - 1, n, k) for o in large.LONG for n, k in ((2048, 384), (1111, 1000), (2300, 513), (5000, 640), (7000, 400))]
    rows += [(o[-1] + 7, len(o) - 1, n, k) for o in GROUPS for n, k in ((1, 1), (70, 130), (300, 257), (129, 1000))]
    assert {f for f, *_ in plan("r", rows)} == {0, 1, 2, 3}
    sums = [(o[-1] + 7, len(o) - 1, m, n) for o, m, n in large.SUMS + [(o, 70, 130) for o in GROUPS]]
    assert {f for f, *_ in plan("s", sums)} == {1, 2, 3}


def test_ranges_cover_k_and_planes_hold_them(plan):
    sizes = [(m, n, k) for m in (1, 65, 300, 1536, 5000) for n in (1, 100, 1000, 4100) for k in (1, 128, 129, 5000, 40000, 131071)]
    for (m, n, k), (form, ranges, each, planes, _, _) in zip(sizes, plan("d", sizes)):
        blocks = (k + 127) // 128
        assert (ranges - 1) * each < blocks <= ranges * each
        assert planes == (0 if ranges == 1 else ranges * m * ((n + 15) // 16 * 16) * 4)
        if form == 3:
            assert m >= 256 and n >= 256 and blocks - (ranges - 1) * each >= 3
        assert planes == oz.oz2_i8_workspace_bytes(m, n, k)


def test_a_last_round_is_left_only_after_whole_ones(plan):
    for (m, n, k), (form, ranges, _, _, tiles, left) in zip(*(lambda s: (s, plan("d", s)))([(256 * a, 256 * b, 2048) for a in range(1, 40, 3) for b in range(1, 40, 5)])):
        if form == 3 and ranges == 1:
            assert left in (0, tiles % 256) and left <= 96 and (left == 0 or tiles > 256)


def test_conversions_take_every_way(plan):
    by_batch = plan("b", [(100, 100, 1), (9000, 16, 1), (9000, 100, 1), (9000, 300, 1), (9000, 1000, 1), (9000, 16384, 1), (900, 20000, 1), (80000, 1000, 8), (2, 1 << 22, 1)])
    assert [p[3] for p in by_batch] == [1] + [0] * 8
    assert {p[0] for p in by_batch} >= {0, 4, 16, 64, 256}
    assert by_batch[-2][1] > 0 and by_batch[-2][2] == 0 and by_batch[4][1] == 0 and by_batch[4][2] > 0     # maxima of columns with the rows, or apart
    assert all(p[4] < 1 << 32 for p in by_batch)
    assert [p[3] for p in plan("q", [(384 * 5, 100, 5), (384 * 5 + 1, 100, 5), (100, 100, 4096)])] == [1, 0, 1]


def test_planes_of_grouped_products(plan):
    sizes = [(rows, groups, n, k) for rows in (1, 100, 5000, 65536) for groups in (1, 2, 9, 500) for n in (1, 100, 1000) for k in (64, 9000)]
    for what, grad in (("r", False), ("s", True)):
        got = plan(what, [(r, g, n, k) if not grad else (r, g, k, n) for r, g, n, k in sizes])
        assert any(ranges > 1 for _, _, ranges, _ in got)
        for (rows, groups, n, k), (form, _, ranges, planes) in zip(sizes, got):
            assert planes == (0 if ranges == 1 else ranges * (groups * k if grad else rows) * ((n + 15) // 16 * 16) * 4)
            assert planes == oz.oz2_i8_grouped_workspace_bytes(rows, n, k, groups, grad) and (ranges == 1 or form in (1, 2))
