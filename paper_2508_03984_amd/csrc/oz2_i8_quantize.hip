// Numbers to 8-bit integers with a binary32 scale for each row of what is written: s = max|x| times the binary32 number next to 1 / 127, rounded to
// nearest, 2^-126 at least, and q the integer next to x / s, ties to even (at most 127: max|x| / s < 127 (1 + 2^-22)).  A row with NaN or an infinity has the scale NaN and zeros.
// (The binary32 number next to 1 / 127 is 2^-28 of it too small, a sixteenth of a unit of the product at most: max|x| / 127 rounded once is another number, one unit up, for 4.7 % of all max|x|.)
//
// q without a division: t = x r with r = 1 / s from the hardware, within a unit of the last place, is within 2^-22 of the quotient (relative), so n = rint(t) is q unless the quotient lies that near to the
// middle of two integers.  e = x - n s, one fused operation, is exact there (a multiple of ulp(s) / 2 below s), so 2 |e| > s says that n is one too far from x, and
// 2 |e| = s that x lies in the middle and the even neighbour is asked for (s / 2 may be subnormal and not exact).  rint is the addition of 1.5 2^23, which leaves q's byte at the end of the word.
//
// Rows are held in registers, so that they are read once; columns need a maximum over all rows before the first byte, so X is read twice where the transpose is wanted.  16384 x 4096 bf16 as it is
// 34 us (5.9 TB/s, X partly from the last-level cache), transposed 66, both 95; 8 of 4096 x 2048 f32 both 123 to 138 us; 100 x 100 both 4.5; 64 x 8192 as it is 3.1 us.  Bound: HBM and, transposed, the conversion's own
// instructions (about 10 a number); the smallest by launch and latency.
#include "oz2_i8_device.hpp"

namespace oz2 {
namespace {

__device__ __forceinline__ float scale_of(float top) { return is_finite(top) ? fmaxf(top * (1.0f / 127.0f), 0x1p-126f) : __builtin_nanf(""); }

// What a scale does to numbers: r = 0 where it is NaN.
struct Scaled {
    float s, r, near;                                         // near: a little below half of s
    __device__ __forceinline__ explicit Scaled(float scale) : s(scale), r(scale < __builtin_inff() ? __builtin_amdgcn_rcpf(scale) : 0.0f), near(0.49999f * scale) {}
};
constexpr float kRint = 12582912.0f;                           // 1.5 2^23

// The bytes of N numbers, four to a word, by S scales in turn for N / S of them each.
template <int N, int S>
__device__ __forceinline__ void quantize(const float (&x)[N], const Scaled (&by)[S], uint32_t (&words)[N / 4]) {
    constexpr int RUN = N / S;
    float t[N];
    bool near = false;
#pragma unroll
    for (int g = 0; g < S; ++g) {
        float off = 0.0f;
#pragma unroll
        for (int i = g * RUN; i < (g + 1) * RUN; i += 2) {
            float e[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                t[i + u] = __builtin_fmaf(x[i + u], by[g].r, kRint);
                e[u] = __builtin_fmaf(kRint - t[i + u], by[g].s, x[i + u]);
            }
            off = fmaxf(fmaxf(off, __builtin_fabsf(e[0])), __builtin_fabsf(e[1]));
        }
        near |= off >= by[g].near;                             // (false for a scale of NaN)
    }
    if (__builtin_expect(__any(near), 0)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Scaled &b = by[i / RUN];
            const float e = __builtin_fmaf(kRint - t[i], b.s, x[i]), twice = 2.0f * __builtin_fabsf(e);
            const bool odd = __builtin_bit_cast(uint32_t, t[i]) & 1;
            if (twice > b.s || (twice == b.s && odd)) t[i] += e > 0.0f ? 1.0f : -1.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        uint32_t w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = __builtin_bit_cast(uint32_t, t[i + u]);
        const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u);
        const uint32_t word = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
        if constexpr (RUN >= 4) words[i / 4] = by[i / RUN].r > 0.0f ? word : 0u;
        else words[i / 4] = (by[i / RUN].r > 0.0f ? word & 0xffffu : 0u) | (by[i / RUN + 1].r > 0.0f ? word & 0xffff0000u : 0u);
    }
}

// 8 numbers of a row of `cols`, from column c on.  `inside`: all of them are there, for the whole wavefront; settle comes when all that a thread reads has been
// asked for, and `none` makes zeros of what was read.
template <int TYPE>
__device__ __forceinline__ void ask(Eight<TYPE> &in, const typename Eight<TYPE>::T *row, int c, int cols, bool inside) {
    if (inside) in.load(row + c);
    else in.load(row + c, cols - c, cols >= 8);
}
template <int TYPE>
__device__ __forceinline__ void settle(Eight<TYPE> &in, int c, int cols, bool inside, bool none) {
    if (!inside || __any(none)) in.move_down(none ? 8 : Eight<TYPE>::down(cols - c, cols >= 8));
}

// The maximum over LANES neighbouring lanes, in all of them, of magnitudes by their bits (which are in the same order, NaN above all).
template <int CONTROL>
__device__ __forceinline__ uint32_t max_moved(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, 0xf, 0xf, true)); }
template <int LANES>
__device__ __forceinline__ float max_over(float magnitude) {
    uint32_t x = __builtin_bit_cast(uint32_t, magnitude) & 0x7fffffffu;
    x = max_moved<0x4e>(max_moved<0xb1>(x));                   // within 4 lanes: [1 0 3 2], [2 3 0 1]
    if constexpr (LANES >= 8) x = max_moved<0x141>(x);         // the halves of 8 lanes mirrored, then of 16
    if constexpr (LANES >= 16) x = max_moved<0x140>(x);
    if constexpr (LANES >= 64) {
        const auto q = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = max((uint32_t)q[0], (uint32_t)q[1]);
        const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = max((uint32_t)h[0], (uint32_t)h[1]);
    }
    return __builtin_bit_cast(float, x);
}

// The scale of a column is the largest of its parts'.
__device__ __forceinline__ void raise_scale(float *scale, float to) { atomicMax(reinterpret_cast<uint32_t *>(scale), __builtin_bit_cast(uint32_t, to)); }

// Row of X for row r of the result, -1 for a row of zeros.
__device__ __forceinline__ int64_t source_row(const I8Quantize &p, int64_t r) {
    if (!p.index) return r;
    const int at = p.index[r];
    return at < 0 || at >= p.x_rows ? -1 : at;
}

// The rows of the result that a call writes as they are: [lo, hi).
__device__ __forceinline__ void rows_written(const I8Quantize &p, int64_t &lo, int64_t &hi) {
    lo = 0;
    hi = p.groups.rows;
    if (p.groups.offsets) {
        lo = min(max(p.groups.offsets[0], 0), p.groups.rows);
        hi = min(p.groups.offsets[p.groups.groups], p.groups.rows);
    }
}

// A row to LANES threads, which hold it, HELD times 8 numbers a thread.  COLUMNS: a workgroup has `each` rows of a group, as many at a time as it has threads for,
// the next ones on their way meanwhile, and raises the scales of the columns by their maxima; else it has one row for every LANES threads.
template <int TYPE, int HELD, int LANES, int THREADS, bool COLUMNS>
__global__ __launch_bounds__(THREADS) void k_i8_rows(I8Quantize p, int each) {
    constexpr int SUBS = THREADS / LANES, WAVES = LANES / 64;
    static_assert(!COLUMNS || THREADS == kI8RowThreads, "");
    __shared__ float tops[2][WAVES > 0 ? WAVES : 1];
    const int sub = (int)threadIdx.x / LANES, me = (int)threadIdx.x % LANES;
    int64_t r, r1;
    float *scales = nullptr;
    if constexpr (COLUMNS) {
        I8Place at;
        if (!i8_find(p.groups, each, 1, blockIdx.x, at)) return;
        r = at.span.lo + (int)at.piece * each + sub;
        r1 = min(at.span.lo + ((int)at.piece + 1) * each, at.span.hi);
        scales = p.scale_t + at.span.group * p.ld_scale_t;
    } else {
        r = (int64_t)blockIdx.x * SUBS + sub;
        r1 = p.groups.rows;
    }
    const int cols = (int)p.cols;
    Eight<TYPE> in[HELD];
    const auto load = [&](int64_t from) {
        const typename Eight<TYPE>::T *const row = static_cast<const typename Eight<TYPE>::T *>(p.X) + max(from, (int64_t)0) * p.ldx;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            ask(in[h], row, (h * LANES + me) * 8, cols, (h + 1) * LANES * 8 <= cols);
        }
    };
    float most[COLUMNS ? HELD : 1][8];
    if constexpr (COLUMNS) {
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < 8; ++i) most[h][i] = 0.0f;
    }
    int64_t from = 0;
    if (r < r1) {
        from = source_row(p, r);
        load(from);
    }
    if constexpr (!COLUMNS) {                                  // (the offsets are read beside the row)
        int64_t lo, hi;
        rows_written(p, lo, hi);
        if (r < lo || r >= hi) return;                         // with LANES > 64 uniform
    }
    for (int turn = 0; r < r1; turn ^= 1) {
        float x[HELD][8], top = 0.0f;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            settle(in[h], (h * LANES + me) * 8, cols, (h + 1) * LANES * 8 <= cols, from < 0);
            in[h].get(x[h]);
        }
        const int64_t here = r;
        r += COLUMNS ? SUBS : r1;
        if (COLUMNS && r < r1) {
            from = source_row(p, r);
            load(from);
        }
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) top = max_magnitude(top, x[h][i], x[h][i + 1]);
            if constexpr (COLUMNS) {
#pragma unroll
                for (int i = 0; i < 8; ++i) most[h][i] = max_magnitude(most[h][i], x[h][i], 0.0f);
            }
        }
        top = max_over<LANES < 64 ? LANES : 64>(top);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) tops[turn][threadIdx.x >> 6] = top;
            __syncthreads();                                   // (nobody writes tops[turn] again before all have met for the next row)
            top = tops[turn][0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) top = max_magnitude(top, tops[turn][w], 0.0f);
        }
        const float s = scale_of(top);
        const Scaled by[1] = {Scaled(s)};
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int c = (h * LANES + me) * 8;
            uint32_t w[2];
            quantize(x[h], by, w);
            if ((c & ~15) < cols) *reinterpret_cast<uint2 *>(p.q + here * p.ld + c) = make_uint2(w[0], w[1]);
        }
        if (me == 0) p.scale[here] = s;
    }
    if constexpr (COLUMNS) {                                   // through LDS, so that 64 lanes raise 64 scales beside each other
        __shared__ __align__(16) float turned[THREADS * 8];
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; i += 4) *reinterpret_cast<f8_v4f *>(turned + threadIdx.x * 8 + i) = f8_v4f{most[h][i], most[h][i + 1], most[h][i + 2], most[h][i + 3]};
            __syncthreads();
            for (int c = (int)threadIdx.x; c < LANES * 8; c += THREADS) {
                float top = turned[c];
#pragma unroll
                for (int u = 1; u < SUBS; ++u) top = max_magnitude(top, turned[u * LANES * 8 + c], 0.0f);
                if (h * LANES * 8 + c < cols) raise_scale(scales + h * LANES * 8 + c, scale_of(top));
            }
        }
    }
}

// Rows of any length, read twice.
template <int TYPE>
__global__ __launch_bounds__(1024) void k_i8_long_rows(I8Quantize p) {
    __shared__ float tops[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r = blockIdx.x;
    int64_t lo, hi;
    rows_written(p, lo, hi);
    if (r < lo || r >= hi) return;
    const int64_t from = source_row(p, r);
    const int cols = (int)p.cols;
    const typename Eight<TYPE>::T *const x_row = static_cast<const typename Eight<TYPE>::T *>(p.X) + max(from, (int64_t)0) * p.ldx;
    const auto get = [&](int c, float(&x)[8]) {
        Eight<TYPE> in;
        in.load(x_row + c, cols - c, cols >= 8);
        in.move_down(from < 0 ? 8 : Eight<TYPE>::down(cols - c, cols >= 8));
        in.get(x);
    };
    float top = 0.0f;
    for (int c = (int)threadIdx.x * 8; c < cols; c += 1024 * 8) {
        float x[8];
        get(c, x);
#pragma unroll
        for (int i = 0; i < 8; i += 2) top = max_magnitude(top, x[i], x[i + 1]);
    }
    top = max_over<64>(top);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    top = 0.0f;
    for (int w = 0; w < 16; ++w) top = max_magnitude(top, tops[w], 0.0f);
    const float s = scale_of(top);
    const Scaled by[1] = {Scaled(s)};
    for (int c = (int)threadIdx.x * 8; c < (cols + 15) / 16 * 16; c += 1024 * 8) {
        float x[8];
        uint32_t w[2];
        get(c, x);
        quantize(x, by, w);
        *reinterpret_cast<uint2 *>(p.q + r * p.ld + c) = make_uint2(w[0], w[1]);
    }
    if (threadIdx.x == 0) p.scale[r] = s;
}

// ------------------------------------------------------------------ transposed
// A scale belongs to a column of a group, so all its rows are read before the first byte is written: the scales grow to their values by
// atomic maxima of their bits (which are in the same order for numbers that are not negative, NaN above all), whatever the order, from 2^-126 on.
__global__ __launch_bounds__(256) void k_i8_least_scales(float *scale, int64_t ld, int cols) {
    const int c = (int)blockIdx.x * 256 + (int)threadIdx.x;
    if (c < cols) scale[(int64_t)blockIdx.y * ld + c] = 0x1p-126f;
}

// `each` rows of a group by LANES * 8 columns, a row to LANES threads.
template <int TYPE, int LANES>
__global__ __launch_bounds__(kI8ColumnThreads) void k_i8_column_scales(I8Quantize p, int each, int parts) {
    constexpr int SUBS = kI8ColumnThreads / LANES, AT_ONCE = 4;
    __shared__ __align__(16) float tops[kI8ColumnThreads * 8];
    I8Place at;
    if (!i8_find(p.groups, each, (uint32_t)parts, blockIdx.x, at)) return;
    const int sub = (int)threadIdx.x / LANES, me = (int)threadIdx.x % LANES;
    const int part = (int)(at.piece % (uint32_t)parts), r0 = at.span.lo + (int)(at.piece / (uint32_t)parts) * each;
    const int r1 = min(r0 + each, at.span.hi), cols = (int)p.cols, c = part * LANES * 8 + me * 8;
    const bool inside = (part + 1) * LANES * 8 <= cols;
    float top[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) top[i] = 0.0f;
    for (int r = r0 + sub; r < r1; r += AT_ONCE * SUBS) {
        Eight<TYPE> in[AT_ONCE];
        int64_t from[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            from[u] = source_row(p, min(r + SUBS * u, r1 - 1)); // (a row twice changes no maximum)
            const typename Eight<TYPE>::T *const row = static_cast<const typename Eight<TYPE>::T *>(p.X) + max(from[u], (int64_t)0) * p.ldx;
            ask(in[u], row, c, cols, inside);
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) settle(in[u], c, cols, inside, from[u] < 0);
#pragma unroll
        for (int u = 0; u < AT_ONCE; u += 2) {
            float x[8], y[8];
            in[u].get(x);
            in[u + 1].get(y);
#pragma unroll
            for (int i = 0; i < 8; ++i) top[i] = max_magnitude(top[i], x[i], y[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; i += 4) *reinterpret_cast<f8_v4f *>(tops + threadIdx.x * 8 + i) = f8_v4f{top[i], top[i + 1], top[i + 2], top[i + 3]};
    __syncthreads();
    for (int i = (int)threadIdx.x; i < LANES * 8; i += kI8ColumnThreads) {
        float most = tops[i];
#pragma unroll
        for (int u = 1; u < SUBS; ++u) most = max_magnitude(most, tops[u * LANES * 8 + i], 0.0f);
        if (part * LANES * 8 + i < cols) raise_scale(p.scale_t + at.span.group * p.ld_scale_t + part * LANES * 8 + i, scale_of(most));
    }
}

// A tile of 128 x 128 of a group: thread (rg, cg) = (t / 16, t % 16) has rows 4 rg + i and columns 8 cg + j, and the bytes of a column change places in LDS, where
// the 16-byte chunk r / 16 of column c is at place (r / 16) ^ (c / 8 % 8).
template <int TYPE>
__global__ __launch_bounds__(kI8TileThreads, 8) void k_i8_turn(I8Quantize p, int tiles) {
    __shared__ __align__(16) uint8_t turned[128 * 128];
    I8Place at;
    if (!i8_find(p.groups, 128, (uint32_t)tiles, blockIdx.x, at)) return;
    const int t = threadIdx.x, rg = t >> 4, cg = t & 15;
    const int tr = (int)(at.piece / (uint32_t)tiles), c0 = (int)(at.piece - (uint32_t)tr * (uint32_t)tiles) * 128;
    const int r0 = at.span.lo + tr * 128, rows = min(128, at.span.hi - r0), cols = (int)p.cols, c = c0 + 8 * cg;
    int64_t source[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) source[i] = r0 + min(4 * rg + i, rows - 1);
    bool empty = false;
    if (p.index) {
        int there[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) there[i] = p.index[source[i]];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            source[i] = there[i] < 0 || there[i] >= p.x_rows ? -1 : there[i];
            empty |= source[i] < 0;
        }
    }
    const bool inside = c0 + 128 <= cols, plain = inside && rows == 128 && !__any(empty);
    const typename Eight<TYPE>::T *const X = static_cast<const typename Eight<TYPE>::T *>(p.X) + c;
    const float *const scale = p.scale_t + at.span.group * p.ld_scale_t;
    Eight<TYPE> in[4];
    float s[8];
    if (inside) {
#pragma unroll
        for (int i = 0; i < 4; ++i) in[i].load(X + max(source[i], (int64_t)0) * p.ldx);
        __builtin_memcpy(s, scale + c, sizeof s);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) in[i].load(X + max(source[i], (int64_t)0) * p.ldx, cols - c, cols >= 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = scale[min(c + j, cols - 1)];
    }
    if (!plain) {
#pragma unroll
        for (int i = 0; i < 4; ++i) in[i].move_down(source[i] < 0 || 4 * rg + i >= rows ? 8 : Eight<TYPE>::down(cols - c, cols >= 8));
    }
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) in[i].get(x[i]);
    uint8_t *const to = turned + 8 * cg * 128 + (rg / 4 ^ (cg & 7)) * 16 + rg % 4 * 4;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const float columns[8] = {x[0][j], x[1][j], x[2][j], x[3][j], x[0][j + 1], x[1][j + 1], x[2][j + 1], x[3][j + 1]};
        const Scaled by[2] = {Scaled(s[j]), Scaled(s[j + 1])};
        uint32_t w[2];
        quantize(columns, by, w);
        *reinterpret_cast<uint32_t *>(to + j * 128) = w[0];
        *reinterpret_cast<uint32_t *>(to + j * 128 + 128) = w[1];
    }
    __syncthreads();
    int8_t *const out = p.qt + (p.side_by_side ? i8_first_col(at.span) : (int64_t)at.span.group * p.cols * p.ldt) + tr * 128;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        const int row = pass * 64 + (t >> 3), chunk = t & 7;
        if (c0 + row < cols && (p.side_by_side || chunk * 16 < rows))
            *reinterpret_cast<f8_v4i *>(out + (int64_t)(c0 + row) * p.ldt + chunk * 16) = *reinterpret_cast<const f8_v4i *>(turned + row * 128 + (chunk ^ (row >> 3 & 7)) * 16);
    }
}

// Everything of a small call in one launch: workgroups from `row_groups` on take 32 columns of a group each, read them for their scales and again for their
// bytes, 64 rows at a time (a row to 4 threads) and 128 in LDS; those before take 4 rows each as they are, of up to 2048 columns.
template <int TYPE>
__global__ __launch_bounds__(256) void k_i8_strips(I8Quantize p, int row_groups, int strips) {
    __shared__ __align__(16) float tops[256 * 8];
    if ((int)blockIdx.x < row_groups) {                        // uniform
        const int lane = threadIdx.x & 63, cols = (int)p.cols;
        const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
        if (r >= p.groups.rows) return;
        const int64_t from = source_row(p, r);
        const typename Eight<TYPE>::T *const row = static_cast<const typename Eight<TYPE>::T *>(p.X) + max(from, (int64_t)0) * p.ldx;
        Eight<TYPE> in[4];
        float x[4][8], top = 0.0f;
#pragma unroll
        for (int h = 0; h < 4; ++h)
            if (h * 512 < cols) ask(in[h], row, h * 512 + lane * 8, cols, (h + 1) * 512 <= cols);
        int64_t lo, hi;
        rows_written(p, lo, hi);
        if (r < lo || r >= hi) return;
#pragma unroll
        for (int h = 0; h < 4; ++h)
            if (h * 512 < cols) {
                settle(in[h], h * 512 + lane * 8, cols, (h + 1) * 512 <= cols, from < 0);
                in[h].get(x[h]);
#pragma unroll
                for (int i = 0; i < 8; i += 2) top = max_magnitude(top, x[h][i], x[h][i + 1]);
            }
        const float s = scale_of(max_over<64>(top));
        const Scaled by[1] = {Scaled(s)};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int c = h * 512 + lane * 8;
            if (h * 512 < cols) {
                uint32_t w[2];
                quantize(x[h], by, w);
                if ((c & ~15) < cols) *reinterpret_cast<uint2 *>(p.q + r * p.ld + c) = make_uint2(w[0], w[1]);
            }
        }
        if (lane == 0) p.scale[r] = s;
        return;
    }
    const int id = (int)blockIdx.x - row_groups, g = id / strips, c0 = (id - g * strips) * 32, cols = (int)p.cols, t = (int)threadIdx.x;
    const int sub = t >> 2, c = c0 + (t & 3) * 8;
    const bool inside = c0 + 32 <= cols;
    const I8Span span = i8_span(p.groups, g);
    const auto row_of = [&](int64_t from) { return static_cast<const typename Eight<TYPE>::T *>(p.X) + max(from, (int64_t)0) * p.ldx; };
    float top[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) top[i] = 0.0f;
    for (int r = span.lo + sub; r < span.hi; r += 256) {
        Eight<TYPE> in[4];
        int64_t from[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) from[u] = source_row(p, min(r + 64 * u, span.hi - 1));  // (a row twice changes no maximum)
#pragma unroll
        for (int u = 0; u < 4; ++u) ask(in[u], row_of(from[u]), c, cols, inside);
#pragma unroll
        for (int u = 0; u < 4; ++u) settle(in[u], c, cols, inside, from[u] < 0);
#pragma unroll
        for (int u = 0; u < 4; u += 2) {
            float x[8], y[8];
            in[u].get(x);
            in[u + 1].get(y);
#pragma unroll
            for (int i = 0; i < 8; ++i) top[i] = max_magnitude(top[i], x[i], y[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; i += 4) *reinterpret_cast<f8_v4f *>(tops + t * 8 + i) = f8_v4f{top[i], top[i + 1], top[i + 2], top[i + 3]};
    __syncthreads();
    {   // 8 threads to a column, 8 rows of threads each
        float most = 0.0f;
        const int column = t >> 3;
#pragma unroll
        for (int u = 0; u < 8; ++u) most = max_magnitude(most, tops[((t & 7) * 8 + u) * 32 + column], 0.0f);
        most = max_over<8>(most);
        const float s = scale_of(most);
        __syncthreads();
        if ((t & 7) == 0) {
            tops[column] = s;
            if (c0 + column < cols) p.scale_t[(int64_t)g * p.ld_scale_t + c0 + column] = s;
        }
    }
    __syncthreads();
    const Scaled by[8] = {Scaled(tops[c - c0]), Scaled(tops[c - c0 + 1]), Scaled(tops[c - c0 + 2]), Scaled(tops[c - c0 + 3]),
                          Scaled(tops[c - c0 + 4]), Scaled(tops[c - c0 + 5]), Scaled(tops[c - c0 + 6]), Scaled(tops[c - c0 + 7])};
    uint8_t *const turned = reinterpret_cast<uint8_t *>(tops + 64);        // [32 columns][128 rows], chunk r / 16 of column c at place (r / 16) ^ (c % 8)
    int8_t *const out = p.qt + (p.side_by_side ? i8_first_col(span) : (int64_t)g * p.cols * p.ldt);
    for (int r0 = span.lo; r0 < span.hi; r0 += 128) {
        const int rows = min(128, span.hi - r0);
        Eight<TYPE> in[2];
        int64_t from[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) from[u] = source_row(p, r0 + min(2 * sub + u, rows - 1));
#pragma unroll
        for (int u = 0; u < 2; ++u) ask(in[u], row_of(from[u]), c, cols, inside);
        float x[2][8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            settle(in[u], c, cols, inside, from[u] < 0 || 2 * sub + u >= rows);
            in[u].get(x[u]);
        }
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float pairs[4] = {x[0][j], x[1][j], x[0][j + 1], x[1][j + 1]};
            const Scaled two[2] = {by[j], by[j + 1]};
            uint32_t w[1];
            quantize(pairs, two, w);
            const int col = c - c0 + j;
#pragma unroll
            for (int u = 0; u < 2; ++u)
                *reinterpret_cast<uint16_t *>(turned + (col + u) * 128 + (sub >> 3 ^ (col + u & 7)) * 16 + (sub & 7) * 2) = (uint16_t)(w[0] >> 16 * u);
        }
        __syncthreads();
        const int row = t >> 3, chunk = t & 7;
        if (c0 + row < cols && (p.side_by_side || chunk * 16 < rows))
            *reinterpret_cast<f8_v4i *>(out + (int64_t)(c0 + row) * p.ldt + (r0 - span.lo) + chunk * 16) =
                *reinterpret_cast<const f8_v4i *>(turned + row * 128 + (chunk ^ (row & 7)) * 16);
        __syncthreads();
    }
}

template <int TYPE, int HELD, int LANES, int THREADS = kI8RowThreads>
hipError_t launch_rows(const I8Quantize &p, int each, hipStream_t stream) {
    if constexpr (THREADS == kI8RowThreads) {
        if (each) {
            hipLaunchKernelGGL((k_i8_rows<TYPE, HELD, LANES, THREADS, true>), dim3((unsigned)i8_quantize_pieces(p.groups, each, 1)), dim3(THREADS), 0, stream, p, each);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((k_i8_rows<TYPE, HELD, LANES, THREADS, false>), dim3((unsigned)f8_ceil(p.groups.rows, THREADS / LANES)), dim3(THREADS), 0, stream, p, 0);
    return hipGetLastError();
}
template <int TYPE, int LANES>
hipError_t launch_columns(const I8Quantize &p, int each, hipStream_t stream) {
    const int64_t parts = f8_ceil(p.cols, LANES * 8);
    hipLaunchKernelGGL((k_i8_column_scales<TYPE, LANES>), dim3((unsigned)i8_quantize_pieces(p.groups, each, parts)), dim3(kI8ColumnThreads), 0, stream, p, each, (int)parts);
    return hipGetLastError();
}

template <int TYPE>
hipError_t launch(const I8Quantize &p, hipStream_t stream) {
    const int64_t cols = p.cols;
    const I8ConvertPlan plan = i8_convert_plan(p);
    if (plan.strips) {
        const int64_t strips = f8_ceil(cols, 32), row_groups = p.q && cols <= kI8StripCols ? f8_ceil(p.groups.rows, 4) : 0;
        hipLaunchKernelGGL((k_i8_strips<TYPE>), dim3((unsigned)(row_groups + strips * p.groups.groups)), dim3(256), 0, stream, p, (int)row_groups, (int)strips);
        if (hipError_t e = hipGetLastError()) return e;
        if (!p.q || row_groups) return hipSuccess;
    } else if (p.qt) {
        const int64_t run = p.side_by_side ? cols : p.groups.groups * cols;      // of scales without a gap
        hipLaunchKernelGGL(k_i8_least_scales, dim3((unsigned)f8_ceil(run, 256), p.side_by_side ? (unsigned)p.groups.groups : 1u), dim3(256), 0, stream, p.scale_t,
                           p.ld_scale_t, (int)run);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (p.q) {
        const int each = plan.rows_each;
        hipError_t e;
        switch (plan.lanes) {
        case 4: e = launch_rows<TYPE, 1, 4>(p, each, stream); break;
        case 16: e = launch_rows<TYPE, 1, 16>(p, each, stream); break;
        case 64: e = launch_rows<TYPE, 1, 64>(p, each, stream); break;
        case 256:
            e = cols <= 2048   ? launch_rows<TYPE, 1, 256>(p, each, stream)
                : cols <= 4096 ? launch_rows<TYPE, 2, 256>(p, each, stream)
                : cols <= 8192 ? launch_rows<TYPE, 4, 256>(p, each, stream)
                               : launch_rows<TYPE, 8, 256>(p, each, stream);
            break;
        case 1024: e = cols <= 8192 ? launch_rows<TYPE, 1, 1024, 1024>(p, 0, stream) : launch_rows<TYPE, 2, 1024, 1024>(p, 0, stream); break;
        default:
            hipLaunchKernelGGL((k_i8_long_rows<TYPE>), dim3((unsigned)p.groups.rows), dim3(1024), 0, stream, p);
            e = hipGetLastError();
        }
        if (e) return e;
    }
    if (!p.qt || plan.strips) return hipSuccess;
    if (plan.columns_each) {
        const int each = plan.columns_each;
        if (hipError_t e = cols <= 32 ? launch_columns<TYPE, 4>(p, each, stream) : cols <= 128 ? launch_columns<TYPE, 16>(p, each, stream)
                                                                                              : launch_columns<TYPE, 64>(p, each, stream)) return e;
    }
    const int64_t tiles = f8_ceil(cols, 128);
    hipLaunchKernelGGL((k_i8_turn<TYPE>), dim3((unsigned)i8_quantize_pieces(p.groups, 128, tiles)), dim3(kI8TileThreads), 0, stream, p, (int)tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_i8_quantize(const I8Quantize &args, int type, hipStream_t stream) {
    return type == kF8Bf16 ? launch<kF8Bf16>(args, stream) : type == kF8F16 ? launch<kF8F16>(args, stream) : launch<kF8F32>(args, stream);
}

}  // namespace oz2
