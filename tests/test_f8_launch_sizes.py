"""Calls at the largest grids, on a stand-in for the HIP runtime that records the launches' sizes: none has 2^32 threads, and a call that would is
refused as unsupported."""
from test_f8_workspace import F8
from test_launch_routes import STAND_IN, run_on_stand_in
from test_workspace_growth import CALLS

SIZES = STAND_IN.replace("int hipLaunchKernel(const void *f, dim3 g, dim3 b, void **a, size_t s, void *st)\n{",
                         "static double most;\ndouble threads(void) { double t = most; most = 0; return t; }\n"
                         "int hipLaunchKernel(const void *f, dim3 g, dim3 b, void **a, size_t s, void *st)\n"
                         "{ double t = (double)g.x * b.x * g.y * b.y * g.z * b.z; if (t > most) most = t;")


def test_the_largest_grids(tmp_path):
    assert "double threads" in SIZES
    got = run_on_stand_in(tmp_path, CALLS.replace("fake.allow.argtypes", "fake.threads.restype = C.c_double\n#") + F8 + r"""
lib.oz2_f8_gated_grad.argtypes = [i64, i64, C.c_int, vp, i64, vp, i64, C.c_int, C.POINTER(M), C.POINTER(M), vp]
lib.oz2_f8_quantize.argtypes = [i64, i64, vp, i64, C.c_int, C.POINTER(M), C.POINTER(M), vp]
wide = M(X, 1 << 23, X, 1 << 16, 1)
out = []
for tiles in (2**22 - 9, 2**22 - 8, 2**22 - 7, 2**22 - 1, 2**22):
    out.append([lib.oz2_f8_gated_grad(128 * tiles, 100, 0, X, 228, X, 100, 0, C.byref(wide), None, None), fake.threads()])
for tiles in (2**23 - 1, 2**23):
    for form in ((None, C.byref(wide)), (C.byref(wide), None)):
        r, c = (128 * tiles, 100) if form[0] else (100, 128 * tiles)
        out.append([lib.oz2_f8_quantize(r, c, X, c, 0, *form, None), fake.threads()])
for rows in (2**12 - 1, 2**12 + 1):                       # blocks of one row, 2^16 of them in a row
    out.append([lib.oz2_f8_quantize(rows, 2**23, X, 2**23, 0, C.byref(wide), None, None), fake.threads()])
for n in (2**27 - 16, 2**27):
    out.append([lib.oz2_ctx_f8_gemm(None, 1, n, 100, 1.0, C.byref(wide), C.byref(wide), 0.0, X, n, 0, None), fake.threads()])
for tiles in (2**24 - 1, 2**24):
    out.append([lib.oz2_ctx_f8_gemm(None, 64 * tiles, 64, 100, 1.0, C.byref(wide), C.byref(wide), 0.0, X, 64, 0, None), fake.threads()])
print(json.dumps(out))
""", SIZES)
    assert all(threads < 2 ** 32 for _, threads in got), got
    assert [status for status, _ in got[:5]] == [0, 0, 2, 2, 2]
    assert all((status == 0) == (threads > 0) and status in (0, 2) for status, threads in got), got
    assert [status for status, _ in got[5:]] == [0, 0, 2, 2, 0, 0, 0, 2, 0, 2]
