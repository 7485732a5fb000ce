"""That the sizes of the GPU tests of 8-bit integers take the forms which those tests are for, by the plans on the CPU: another fit of the plans must not leave a form untested."""
from test_i8_forms import plan  # noqa: F401"""That the sizes of the GPU tests of 8-bit integers take the forms which those tests are for, by the plans on the CPU: another fit of the plans must not leave a form untested."""
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