"""Memory for the planes of K ranges of 8-bit floating-point products, on the CPU: the library runs in a process of its own on a stand-in for the
HIP runtime whose allocations can be refused, in which way can be said, and whose current device can be changed."""
import json
import re

import pytest

from test_launch_routes import STAND_IN, run_on_stand_in
from test_workspace_growth import CALLS, MEMORY

OWN = r"""
static int refusal = 2, device;
void refuse_with(int code) { refusal = code; }
void use_device(int d) { device = d; }
int hipGetDevice(int *d) { *d = device; return 0; }
int hipSetDevice(int d) { device = d; return 0; }
"""
F8 = r"""
class M(C.Structure):
    _fields_ = [("q", vp), ("ld", i64), ("scale", vp), ("ld_scale", i64), ("block_rows", C.c_int)]
lib.oz2_ctx_f8_gemm.argtypes = [vp, i64, i64, i64, C.c_float, C.POINTER(M), C.POINTER(M), C.c_float, vp, i64, C.c_int, vp]
lib.oz2_ctx_f8_gated.argtypes = [vp, i64, i64, i64, C.c_int, C.POINTER(M), C.POINTER(M), vp, i64, vp, i64, C.c_int, vp]
lib.oz2_f8_workspace_bytes.argtypes = [i64, i64, i64, C.c_int]
lib.oz2_f8_workspace_bytes.restype = sz
lib.oz2_ctx_stage_ptr.argtypes = [vp, C.c_int, C.POINTER(vp), C.POINTER(i64)]
lib.oz2_ctx_set_workspace.argtypes = [vp, vp, sz]
lib.oz2_ctx_release.argtypes = [vp]

def f8(c, m, n, k, gated=False, allow=2**63):
    # (status, in K ranges?, allocations asked for, buffers freed)
    mat = M(X, (k + 15) // 16 * 16, X, (k + 511) // 512 * 4, 1)
    fake.forget(); fake.allow(allow)
    asked, freed = fake.times_asked(), fake.times_freed()
    if gated:
        status = lib.oz2_ctx_f8_gated(c, m, n, k, 0, C.byref(mat), C.byref(mat), X, n, None, 0, 0, None)
    else:
        status = lib.oz2_ctx_f8_gemm(c, m, n, k, 1.0, C.byref(mat), C.byref(mat), 0.0, X, n, 0, None)
    names = fake.launched().decode().split("\n")[:-1]
    return [status, any("k_f8_ranges" in x for x in names), fake.times_asked() - asked, fake.times_freed() - freed, len(names)]

def need(m, n, k, gated=False):
    return lib.oz2_f8_workspace_bytes(m, n, k, int(gated))

def stage(c):
    p, d = vp(), (i64 * 4)()
    return [lib.oz2_ctx_stage_ptr(c, 0, C.byref(p), d), p.value, list(d)]
"""
SMALL, LONG, LONGER = (150, 140, 20000), (1536, 1000, 40000), (3000, 3000, 1 << 20)


def on_stand_in(d, body, data=None):
    base = re.sub(r"int (hipMalloc|hipFree|hipGetLastError|hipGetDevice|hipSetDevice)\(.*\n", "", STAND_IN)
    memory = MEMORY.replace("last_error = 2", "last_error = refusal")
    assert memory != MEMORY
    head = "SMALL, LONG, LONGER = %r, %r, %r\n" % (SMALL, LONG, LONGER)
    return run_on_stand_in(d, CALLS + F8 + head + body, base + OWN + memory, data=json.dumps(data))


def test_a_product_leaves_the_buffer_of_other_products_alone(tmp_path):
    """A captured graph may hold the buffer that a DGEMM has run in: planes do not take its place, and its stages stay."""
    got = on_stand_in(tmp_path, r"""
assert 0 < need(*SMALL) < need(*LONG) < need(*LONGER)
c = context()
assert call(c, 64, 64, 64, 14)[0] == 0
before = stage(c)
print(json.dumps([before, [f8(c, *s) + [stage(c)] for s in (SMALL, LONG, LONGER, (150, 70, 20000, True), SMALL, LONGER)]]))
""")
    before, calls = got
    assert before[0] == 0 and before[1]
    for status, ranges, asked, freed, launches, stage in calls:
        assert status == 0 and ranges and freed == 0 and launches == 2 and stage == before
    assert [c[2] for c in calls[:3]] == [1, 1, 1] and [c[2] for c in calls[4:]] == [0, 0]


def test_planes_stay_where_they_are(tmp_path):
    """A captured graph may hold them: neither larger planes nor a DGEMM that needs a larger buffer free them, and they go with the context's memory."""
    got = on_stand_in(tmp_path, r"""
c = context()
out = [f8(c, *s) for s in (SMALL, LONG, LONGER)]
freed = fake.times_freed()
status = [call(c, n, n, n, 14)[0] for n in (64, 300, 1000, 4000)]
by_dgemm = fake.times_freed() - freed
out += [f8(c, *s) for s in (SMALL, LONG, LONGER)]
freed = fake.times_freed()
assert lib.oz2_ctx_release(c) == 0
released = fake.times_freed() - freed
out += [f8(c, *SMALL)]
freed = fake.times_freed()
lib.oz2_destroy(c)
print(json.dumps([out, status, by_dgemm, released, fake.times_freed() - freed]))
""")
    calls, status, by_dgemm, released, destroyed = got
    assert [c[:4] for c in calls] == [[0, True, 1, 0]] * 3 + [[0, True, 0, 0]] * 3 + [[0, True, 1, 0]]
    assert status == [0] * 4 and by_dgemm == 3                # its own three smaller ones
    assert released == 4 and destroyed == 1


def test_few_buffers_however_sizes_come(tmp_path):
    """Growing sizes: a new buffer is twice as large as the one before, so there are few, and all together are less than twice the largest."""
    got = on_stand_in(tmp_path, r"""
c = context()
sizes = sorted((need(m, 1000, 40000), m) for m in range(70, 4000, 10) if need(m, 1000, 40000))
out = [f8(c, m, 1000, 40000) for _, m in sizes]
print(json.dumps([len(out), [o[:2] + o[3:4] for o in out], sum(o[2] for o in out)]))
""")
    n, calls, asked = got
    assert n > 100 and all(c == [0, True, 0] for c in calls)
    assert asked <= 12


@pytest.mark.parametrize("gated", [False, True])
def test_refused(tmp_path, gated):
    """Out of memory: one range.  Another error (a stream that is being captured allows no allocation): reported, and nothing launched."""
    got = on_stand_in(tmp_path, r"""
gated = json.loads(sys.stdin.read())
out = []
for code in (2, 900):
    c = context()
    assert call(c, 64, 64, 64, 14)[0] == 0
    before = stage(c)
    fake.refuse_with(code)
    refused = f8(c, *LONG, gated, allow=4096)
    again = call(c, 64, 64, 64, 14)[0]
    fake.refuse_with(2)
    out.append([refused, stage(c) == before, again, f8(c, *LONG, gated)])
print(json.dumps(out))
""", data=gated)
    (memory, kept, again, then), (other, kept_too, again_too, then_too) = got
    assert memory[:2] == [0, False] and memory[4] == 1 and memory[3] == 0
    assert other[0] == 4 and other[3:] == [0, 0]
    assert kept and kept_too and again == again_too == 0
    assert then[:3] == then_too[:3] == [0, True, 1]


def test_only_as_much_as_there_is(tmp_path):
    """What is refused in twice the size of the last buffer may be had in its own."""
    got = on_stand_in(tmp_path, r"""
c = context()
sizes = sorted((need(m, n, 40000), m, n) for m in range(100, 4000, 100) for n in (300, 1000, 1500))
(one, *first), (two, *larger) = next((a, b) for a in sizes for b in sizes if a[0] > 2**24 and a[0] + 2**22 < b[0] < 2 * a[0] - 2**22)
a = f8(c, *first, 40000)
print(json.dumps([a, f8(c, *larger, 40000, allow=two), f8(c, *larger, 40000)]))
""")
    assert got[0][:4] == [0, True, 1, 0]
    assert got[1][:4] == [0, True, 2, 0] and got[2][:4] == [0, True, 0, 0]


def test_limits(tmp_path):
    """A limit holds for all that the context has; what it refuses costs nothing that was there.  A DGEMM goes before planes."""
    got = on_stand_in(tmp_path, r"""
out = []
for limit in (need(*LONG) - 1, need(*LONG) + 2**24):
    c = context()
    lib.oz2_ctx_set_workspace_limit(c, limit)
    s = call(c, 64, 64, 64, 2)[0]
    before = stage(c)
    out.append([s, f8(c, *LONG), stage(c) == before])
    lib.oz2_destroy(c)
c = context()
lib.oz2_ctx_set_workspace_limit(c, need(*LONG))           # no more than the planes, and they come first
first = f8(c, *LONG)
then = f8(c, *LONG)
freed = fake.times_freed()
s = call(c, 64, 64, 64, 2)[0]
out.append([first, then, s, fake.times_freed() - freed, f8(c, *LONG), f8(c, *SMALL)])
lib.oz2_ctx_set_workspace_limit(c, 1024)
out.append(f8(c, *SMALL))
print(json.dumps(out))
""")
    below, above, first, lowered = got
    assert below == [0, [0, False, 0, 0, 1], True]
    assert above[0] == 0 and above[2] and above[1][1] in (False, True) and above[1][3] == 0
    assert first[0][:4] == [0, True, 1, 0] and first[1][:4] == [0, True, 0, 0]
    assert first[2] == 0 and first[3] == 1                    # the planes make room
    assert first[4][:4] == [0, False, 0, 0]
    assert lowered[:4] == [0, False, 0, 0]


def test_a_callers_buffer(tmp_path):
    """Planes lie in it if it has room, over the stages of the product before, which then are no more to be had; nothing is allocated."""
    got = on_stand_in(tmp_path, r"""
c = context()
f8(c, *LONG)
freed = fake.times_freed()
assert lib.oz2_ctx_set_workspace(c, 1 << 30, 2**26) == 0
given = fake.times_freed() - freed
assert call(c, 64, 64, 64, 14)[0] == 0
before = stage(c)
too_large = f8(c, *LONGER) + [stage(c) == before]
fits = f8(c, *SMALL) + stage(c)[:1]
print(json.dumps([given, before, too_large, fits]))
""")
    given, before, too_large, fits = got
    assert given == 1 and before[0] == 0
    assert too_large == [0, False, 0, 0, 1, True]
    assert fits == [0, True, 0, 0, 2, 1]


def test_devices(tmp_path):
    """Planes on the device that is current, and again the same ones on the first device."""
    got = on_stand_in(tmp_path, r"""
c = context()
out = []
for d in (0, 1, 0, 1):
    fake.use_device(d)
    out.append(f8(c, *LONG))
freed = fake.times_freed()
lib.oz2_destroy(c)
d = C.c_int(-1)
fake.hipGetDevice(C.byref(d))
print(json.dumps([out, fake.times_freed() - freed, d.value]))
""")
    assert [o[:4] for o in got[0]] == [[0, True, 1, 0]] * 2 + [[0, True, 0, 0]] * 2
    assert got[1:] == [2, 1]
