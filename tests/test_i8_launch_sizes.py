"""8-bit integer calls at the largest grids, on a stand-in for the HIP runtime that records the launches' sizes: none has 2^32 threads or more than 65535 workgroups
in its second dimension, and a call that would is refused as unsupported before anything is launched."""
from test_f8_launch_sizes import SIZES
from test_launch_routes import run_on_stand_in
from test_workspace_growth import CALLS


def test_the_largest_grids(tmp_path):
    stand_in = SIZES.replace("static double most;", "static double most, second;\ndouble rows(void) { double t = second; second = 0; return t; }\n").replace(
        "double t = (double)g.x", "if (g.y > second) second = g.y; double t = (double)g.x")
    assert "double rows" in stand_in and "second = g.y" in stand_in
    got = run_on_stand_in(tmp_path, CALLS.replace("fake.allow.argtypes", "fake.threads.restype = fake.rows.restype = C.c_double\n#") + r"""
class M(C.Structure):
    _fields_ = [("q", vp), ("ld", i64), ("scale", vp), ("ld_scale", i64)]
P, flt, ci = C.POINTER(M), C.c_float, C.c_int
lib.oz2_i8_quantize.argtypes = [i64, i64, i64, vp, i64, ci, P, P, vp]
lib.oz2_i8_quantize_grouped.argtypes = [i64, i64, vp, i64, i64, ci, vp, i64, vp, P, P, vp]
lib.oz2_i8_gemm.argtypes = [i64, i64, i64, flt, P, P, flt, vp, i64, ci, vp]
lib.oz2_i8_grouped_gemm.argtypes = lib.oz2_i8_grouped_grad.argtypes = [i64, i64, i64, i64, vp, flt, P, P, flt, vp, i64, ci, vp]
wide = C.byref(M(X, 1 << 23, X, 1 << 30))
out = []
def note(status):
    out.append([status, fake.threads(), fake.rows()])
big = [1, 5, 600, 70000, 2**20, 2**23, 2**24 - 1, 2**24, 2**26 + 1, 2**28, 2**30]
for a in big:
    for b in big:
        for t in range(3):
            if b <= 2**23:
                note(lib.oz2_i8_quantize(1, a, b, X, b, t, wide, None, None))
            if a <= 2**23:
                note(lib.oz2_i8_quantize(1, a, b, X, b, t, None, wide, None))
            if a <= 2**23 and b <= 2**23:
                for batch in (3, 5000, 2**20):
                    note(lib.oz2_i8_quantize(batch, a, b, X, b, t, wide, wide, None))
        for groups in (1, 3, 64, 4096):
            if a // 128 * 128 + 128 * groups <= 2**23 and b <= 2**23:
                note(lib.oz2_i8_quantize_grouped(a, b, X, a, b, 0, None, groups, X, wide, wide, None))
            if a // 128 * 128 + 128 * groups <= 2**23:
                note(lib.oz2_i8_quantize_grouped(a, b, X, a, b, 0, X, groups, X, None, wide, None))
                note(lib.oz2_i8_grouped_grad(b, 300, a, groups, X, 1.0, wide, wide, 0.0, X, 300, 0, None))
            for k in (100, 5000):
                note(lib.oz2_i8_grouped_gemm(a, b, k, groups, X, 1.0, wide, wide, 0.0, X, b, 0, None))
        for k in (100, 5000, 131071):
            note(lib.oz2_i8_gemm(a, b, k, 1.0, wide, wide, 0.0, X, b, 0, None))
print(json.dumps(out))
""", stand_in)
    assert len(got) > 2000 and {status for status, _, _ in got} == {0, 2}
    assert all(threads < 2 ** 32 and rows <= 65535 for _, threads, rows in got), max(got, key=lambda x: x[1])
    assert all((status == 0) == (threads > 0) for status, threads, _ in got)
    assert sum(status == 0 for status, _, _ in got) > 1000
