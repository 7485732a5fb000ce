"""The stages of the last product, after a call that gave up its buffer: they are refused, not somewhere else.  On the CPU, on a stand-in for the HIP
runtime whose allocations can be refused."""
from test_f8_workspace import on_stand_in


def test_after_a_refused_growth(tmp_path):
    got = on_stand_in(tmp_path, r"""
c = context()
assert call(c, 64, 64, 64, 14)[0] == 0
before = stage(c)
refused = call(c, 2000, 2000, 2000, 14, allow=4096)
after = stage(c)
again = call(c, 64, 64, 64, 14)
print(json.dumps([before, refused, after, again[0], stage(c)]))
""")
    before, refused, after, again, then = got
    assert before[0] == 0 and refused == [3, []]
    assert after[:2] == [1, None]
    assert again == 0 and then[0] == 0 and then[2] == before[2]


def test_after_a_prepared_product_moved_the_buffer(tmp_path):
    """A refused growth of a product of prepared operands, and one that is not refused."""
    got = on_stand_in(tmp_path, r"""
out = []
for allow in (4096, 2**63):
    c = context()
    assert call(c, 64, 64, 64, 14)[0] == 0
    status = prepared(c, 2000, 2000, 2000, 14, allow=allow)[0]
    out.append([status] + stage(c)[:2])
print(json.dumps(out))
""")
    assert got == [[3, 1, None], [0, 1, None]]


def test_after_a_limit_that_refuses(tmp_path):
    """Nothing was given up: the stages are where they were."""
    got = on_stand_in(tmp_path, r"""
c = context()
assert call(c, 64, 64, 64, 14)[0] == 0
before = stage(c)
lib.oz2_ctx_set_workspace_limit(c, 65536)
refused = call(c, 2000, 2000, 2000, 14)
print(json.dumps([refused, stage(c) == before]))
""")
    assert got == [[3, []], True]
