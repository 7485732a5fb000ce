"""That the sizes of the GPU tests of 8-bit integers take the forms which those tests are for, by the plans on the CPU: another fit of the plans must not leave a form untested."""
from test_i8_forms import plan  # noqa: F401


def conversions(plan, batches, grouped):  # noqa: F811
    got = plan("b", [(b * r, c, b) for b, r, c in batches]) if batches else []
    return got + (plan("q", [(o[-1] + 9, c, len(o) - 1) for o, c in grouped]) if grouped else [])


def test_conversions_take_every_form(plan):  # noqa: F811
    import test_gpu_i8_conversions as T

    def held(cols):                                            # times 8 numbers that each of 256 threads holds of a row
        return -(-cols // 2048)

    for batches, grouped in ((T.TOGETHER, []), ([], T.GROUPED_TOGETHER)):
        got = conversions(plan, batches, grouped)
        assert all(rows_each > 0 and columns_each == 0 and not strips for _, rows_each, columns_each, strips, _ in got)
        cols = [c for *_, c in batches + grouped]
        assert {(p[0], held(c)) for p, c in zip(got, cols)} == {(4, 1), (16, 1), (64, 1), (256, 1), (256, 2), (256, 3), (256, 5)}    # (3 and 5: as 4 and 8)
        # several rows one after the other for a thread
        assert all(any(p[0] == lanes and p[1] > 256 // lanes for p in got) for lanes in ((4, 16, 64, 256) if batches else (64, 256)))
    for batches, grouped in ((T.APART, []), ([], T.GROUPED_APART)):
        got = conversions(plan, batches, grouped)
        assert all(rows_each == 0 and columns_each > 0 and not strips for _, rows_each, columns_each, strips, _ in got)
        cols = [c for *_, c in batches + grouped]
        assert {4 if c <= 32 else 16 if c <= 128 else 64 for c in cols} == {4, 16, 64}
        if batches:
            assert {(p[0], held(c) if p[0] == 256 else 0) for p, c in zip(got, cols)} == {(4, 0), (16, 0), (64, 0), (256, 1), (256, 2), (256, 3), (256, 5), (0, 0)}
    assert all(p[3] for p in conversions(plan, [], T.GROUPED_STRIPS))
    # a row to 1024 threads, which hold 8 or 16 numbers of it, and rows read twice, where the transpose goes in one launch
    from test_gpu_i8 import SIZES
    lanes = {(p[0], c > 8192) for p, (_, c) in zip(plan("b", [(r, c, 1) for r, c in SIZES]), SIZES) if p[3]}
    assert {(1024, False), (1024, True), (0, True)} <= lanes


def test_many_groups_take_large_tiles(plan):  # noqa: F811
    import test_gpu_i8_many_groups as T
    for what, sizes in (("r", T.ROWS), ("s", T.SUMS)):
        got = plan(what, [(T.offsets_of(g, mean)[-1] + 7, g, a, b) for g, mean, a, b in sizes])
        assert [(form, ranges) for form, _, ranges, _ in got] == [(3, 1)] * len(sizes), got
        for groups, mean, *_ in sizes:
            of = T.lengths(groups, mean)
            assert min(of) == 0 and of.count(0) < groups / 4 and (groups < 67 or of[62:67] == [0, 300, 0, 259, 1])
            assert what == "r" or any(0 < n <= 256 for n in of)  # (which are left to smaller tiles)


def span(offsets, g, rows):
    """The rows that a group is taken to have, whatever the offsets are."""
    lo = min(max(offsets[g], 0), rows)
    return lo, min(max(offsets[g + 1], lo), rows)


def test_bad_offsets_meet_every_form_and_stay_inside(plan):  # noqa: F811
    import test_gpu_i8_bad_offsets as T
    rows = [(form, ranges > 1) for form, _, ranges, _ in plan("r", T.ROWS)]
    assert rows == [(0, False), (1, False), (2, False), (3, False), (3, False), (1, True)], rows
    sums = [(form, ranges > 1) for form, _, ranges, _ in plan("s", T.SUMS)]
    assert sums == [(1, False), (2, False), (3, False), (3, False), (1, True)], sums
    got = plan("q", [(r, c, g) for r, g, c in T.CONVERSIONS])
    assert [(p[3], p[1] > 0, p[2] > 0) for p in got] == [(1, 0, 0), (0, 1, 0), (0, 1, 0), (0, 0, 1), (0, 0, 1)], got
    left = []
    for n_rows, groups, n, _ in T.ROWS[3:5]:                   # of large tiles: those that a last round leaves to smaller ones, on 256 units
        for bad in T.bad_offsets(n_rows, groups):
            units = sum(-(-(hi - lo) // 256) for lo, hi in (span(bad, g, n_rows) for g in range(groups)))
            share = (units * -(-n // 256) + 7) // 8
            left.append(share % 32 if share > 32 and share % 32 <= 12 else 0)
    assert any(left)
    for n_rows, groups, *_ in T.ROWS + T.SUMS + T.CONVERSIONS:
        wide = n_rows // 128 * 128 + 128 * groups
        for bad in T.bad_offsets(n_rows, groups):
            for g in range(groups):
                lo, hi = span(bad, g, n_rows)
                assert 0 <= lo <= hi <= n_rows and (lo // 128 + g) * 128 + (hi - lo + 127) // 128 * 128 <= wide


def test_overflows_and_far_operands_meet_every_form(plan):  # noqa: F811
    import test_gpu_i8_far_large as F
    import test_gpu_i8_overflow as T
    got = plan("d", T.PRODUCTS + [(F.ROWS, F.N, F.K), (F.N, F.ROWS, F.K)])
    assert [(p[0], p[1] > 1) for p in got] == [(0, False), (1, False), (2, False), (3, False), (1, True), (3, True), (3, False), (3, False)], got
    got = plan("r", [(o[-1] + 2, len(o) - 1, n, k) for o, n, k in T.ROWS])
    assert [(form, ranges > 1) for form, _, ranges, _ in got] == [(0, False), (1, False), (2, False), (1, True), (3, False)], got
    got = plan("s", [(o[-1] + 2, len(o) - 1, m, n) for o, m, n in T.SUMS] + [(F.TOKENS, 2, F.M, F.N), (F.TOKENS, 2, F.N, F.M)])
    assert [(form, ranges > 1) for form, _, ranges, _ in got] == [(1, False), (2, False), (1, True), (3, False), (3, False), (3, False)], got


def test_the_check_of_overflows_passes_over_nothing():
    import pytest
    import torch
    import test_gpu_i8_overflow as T
    want = torch.tensor([[1.0, 1e6, -1e6, 65510.0]], dtype=torch.float64)
    right = torch.tensor([[1.0, float("inf"), -float("inf"), 65504.0]], dtype=torch.float16)
    T.check(right, want, want)
    for i, wrong in ((1, 0.0), (1, 65504.0), (1, -float("inf")), (2, float("inf")), (3, float("inf")), (0, float("inf")), (0, 1.01), (1, float("nan"))):
        bad = right.clone()
        bad[0, i] = wrong
        with pytest.raises(AssertionError):
            T.check(bad, want, want)
