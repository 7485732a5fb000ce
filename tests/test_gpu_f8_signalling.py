"""Conversion to 8-bit floating point beside signalling NaN, which maxima of the hardware may answer with the smaller number: the scale covers the
finite numbers of the block all the same, to the bit.  Made from bits, since a conversion would quiet them."""
import numpy as np
import pytest

import f8_reference as R

torch = pytest.importorskip("torch")
import paper_2508_03984_amd as oz  # noqa: E402
from test_gpu_f8 import DTYPES, host  # noqa: E402

pytestmark = pytest.mark.gpu
WORD = {"bf16": np.int16, "f16": np.int16, "f32": np.int32}
# Words that are NaN with the first bit of the fraction clear, of either sign; quiet NaN; infinity.
SIGNALLING = {"bf16": [0x7F81, 0xFF81, 0x7FBF], "f16": [0x7C01, 0xFC01, 0x7DFF], "f32": [0x7F800001, 0xFF800001, 0x7FBFFFFF]}
QUIET = {"bf16": 0x7FC0, "f16": 0x7E00, "f32": 0x7FC00000}
INFINITE = {"bf16": 0x7F80, "f16": 0x7C00, "f32": 0x7F800000}


def with_bits(x, dtype, places):
    """x as a tensor of dtype, with the words of `places`, (row, column, bits)."""
    words = torch.from_numpy(x).to(DTYPES[dtype]).view(torch.int16 if dtype != "f32" else torch.int32).numpy().copy()
    for r, c, bits in places:
        words[r, c] = np.array(bits, np.int64).astype(WORD[dtype])
    return torch.from_numpy(words).cuda().view(DTYPES[dtype])


def check(X, block_rows):
    rows, cols = X.shape
    seen = host(X)
    for as_is, transposed in ((1, 1), (1, 0), (0, 1)):
        a, t = oz.F8.empty(rows, cols, block_rows), oz.F8.empty(cols, rows, block_rows)
        oz.oz2_f8_quantize(rows, cols, X, cols, a if as_is else None, t if transposed else None)
        for out, asked, of in ((a, as_is, seen), (t, transposed, seen.T)):
            if not asked:
                continue
            want_q, want_s = R.quantize(of, block_rows)
            assert np.array_equal(host(out.scale), want_s)
            q, nan = host(out.q), (want_q & 127) == 127
            assert np.array_equal((q & 127) == 127, nan) and np.array_equal(q[~nan], want_q[~nan])


def spread(rng, rows, cols):
    return np.clip(rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, cols))), -6e4, 6e4)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols", [(128, 128), (131, 200), (9, 8)])
def test_one_in_every_row(rows, cols, dtype, block_rows):
    """At every place of a block once, whatever a thread or a lane has before and after it."""
    rng = np.random.default_rng(rows + cols)
    for kind in range(3):
        x = spread(rng, rows, cols)
        check(with_bits(x, dtype, [(r, (r + kind) % cols, SIGNALLING[dtype][kind]) for r in range(rows)]), block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_behind_the_largest(dtype, block_rows):
    """Numbers that fall along a row and along a column: whatever comes after the NaN is smaller than what came before it."""
    falling = 2.0 ** -np.arange(12)[np.minimum(np.arange(130) % 16, 11)] * 100
    x = falling[:, None] * falling[None, :] / 100
    for place in range(20):
        bits = SIGNALLING[dtype][place % 3]
        check(with_bits(x, dtype, [(0, place, bits)]), block_rows)
        check(with_bits(x, dtype, [(place, 0, bits)]), block_rows)
        check(with_bits(x[:1], dtype, [(0, place, bits)]), block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_among_quiet_ones_and_infinities(dtype, block_rows):
    rng = np.random.default_rng(5)
    rows, cols = 300, 260
    x = spread(rng, rows, cols)
    kinds = [*SIGNALLING[dtype], QUIET[dtype], INFINITE[dtype]]
    places = [(int(r), int(c), kinds[i % len(kinds)]) for i, (r, c) in enumerate(zip(rng.integers(0, rows, 4000), rng.integers(0, cols, 4000)))]
    places += [(7, c, kinds[c % len(kinds)]) for c in range(cols)] + [(r, 9, kinds[r % len(kinds)]) for r in range(rows)]
    check(with_bits(x, dtype, places), block_rows)
    check(with_bits(x, dtype, [(r, c, kinds[(r + c) % len(kinds)]) for r in range(rows) for c in range(cols)]), block_rows)
