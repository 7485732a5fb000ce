// Numbers to 8-bit integers with a binary32 scale for each row of what is written: s = max|x| times the binary32 number next to 1 / 127, rounded to
// nearest, 2^-126 at least, and q the integer next to x / s, ties to even (at most 127: max|x| / s < 127 (1 + 2^-22)).  A row with NaN or an infinity has the scale NaN and zeros.
//
// q without a division per number: t = x r with r = 1 / s rounded is within 3 2^-24 of the quotient, so n = rint(t) is q unless the quotient lies that near to the
// middle of two integers.  e = x - n s, one fused operation, is exact there (a multiple of ulp(s) / 2 below s), so 2 |e| > s says that n is one too far from x, and
// 2 |e| = s that x lies in the middle and the even neighbour is asked for (s / 2 may be subnormal and not exact).  rint is the addition of 1.5 2^23, which leaves q's byte at the end of the word.
#include "oz2_i8_device.hpp"

namespace oz2 {
namespace {

__device__ __forceinline__ float scale_of(float top) { return is_finite(top) ? fmaxf(top * (1.0f / 127.0f), 0x1p-126f) : __builtin_nanf(""); }

// What a scale does to numbers: r = 0 where it is NaN.
struct Scaled {
    float s, r, near;                                         // near: a little below half of s
    __device__ __forceinline__ explicit Scaled(float scale) : s(scale), r(scale < __builtin_inff() ? 1.0f / scale : 0.0f), near(0.49999f * scale) {}
};
constexpr float kRint = 12582912.0f;                           // 1.5 2^23

// The bytes of 4 numbers, with a scale for each or one for all.
template <int N>
__device__ __forceinline__ uint32_t quantize4(const float (&x)[4], const Scaled (&by)[N]) {
    float t[4], n[4], e[4];
    bool near = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Scaled &b = by[N == 1 ? 0 : i];
        t[i] = __builtin_fmaf(x[i], b.r, kRint);
        n[i] = t[i] - kRint;
        e[i] = __builtin_fmaf(-n[i], b.s, x[i]);
        near |= __builtin_fabsf(e[i]) >= b.near;               // (false for a scale of NaN)
    }
    if (__builtin_expect(near, 0)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Scaled &b = by[N == 1 ? 0 : i];
            const float off = 2.0f * __builtin_fabsf(e[i]);
            const bool odd = __builtin_bit_cast(uint32_t, t[i]) & 1;
            if (off > b.s || (off == b.s && odd)) t[i] += e[i] > 0.0f ? 1.0f : -1.0f;
        }
    }
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = by[N == 1 ? 0 : i].r > 0.0f ? __builtin_bit_cast(uint32_t, t[i]) : 0u;
    const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// Row of X for row r of the result, -1 for a row of zeros.
__device__ __forceinline__ int64_t source_row(const I8Quantize &p, int64_t r) {
    if (!p.index) return r;
    const int at = p.index[r];
    return at < 0 || at >= p.x_rows ? -1 : at;
}

__device__ __forceinline__ float wave_max(float x) {           // of what is not NaN-free: v_maximum3 keeps it
#pragma unroll
    for (int by = 32; by > 0; by /= 2) x = max_magnitude(x, __shfl_xor(x, by), 0.0f);
    return x;
}

// A row to 256 threads (ALONE: to a wavefront), which hold it, HELD times 8 numbers a thread.
template <int TYPE, int HELD, bool ALONE>
__global__ __launch_bounds__(kI8RowThreads) void k_i8_rows(I8Quantize p) {
    __shared__ float tops[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    constexpr int THREADS = ALONE ? 64 : kI8RowThreads;
    const int me = ALONE ? lane : (int)threadIdx.x;
    const int64_t r = ALONE ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    int64_t lo = 0, hi = p.groups.rows;
    if (p.groups.offsets) {
        lo = min(max(p.groups.offsets[0], 0), p.groups.rows);
        hi = min(p.groups.offsets[p.groups.groups], p.groups.rows);
    }
    if (r < lo || r >= hi) return;                             // uniform (over the wavefront if it has a row of its own)
    const int64_t from = source_row(p, r);
    const int cols = (int)p.cols;
    const typename Eight<TYPE>::T *const x_row = static_cast<const typename Eight<TYPE>::T *>(p.X) + max(from, (int64_t)0) * p.ldx;
    Eight<TYPE> in[HELD];
    float top = 0.0f;
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        const int c = (h * THREADS + me) * 8;
        if (c + 8 <= cols) in[h].load(x_row + c);
        else in[h].load(x_row + c, cols - c, cols >= 8);
    }
    float x[HELD][8];
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        const int c = (h * THREADS + me) * 8;
        in[h].move_down(from < 0 ? 8 : Eight<TYPE>::down(cols - c, cols >= 8));
        in[h].get(x[h]);
#pragma unroll
        for (int i = 0; i < 8; i += 2) top = max_magnitude(top, x[h][i], x[h][i + 1]);
    }
    top = wave_max(top);
    if (!ALONE) {
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = max_magnitude(max_magnitude(tops[0], tops[1], tops[2]), tops[3], 0.0f);
    }
    const float s = scale_of(top);
    const Scaled by[1] = {Scaled(s)};
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        const int c = (h * THREADS + me) * 8;
        const float a[4] = {x[h][0], x[h][1], x[h][2], x[h][3]}, b[4] = {x[h][4], x[h][5], x[h][6], x[h][7]};
        if ((c & ~15) < cols) *reinterpret_cast<uint2 *>(p.q + r * p.ld + c) = make_uint2(quantize4(a, by), quantize4(b, by));
    }
    if (me == 0) p.scale[r] = s;
}

// Rows of any length, read twice.
template <int TYPE>
__global__ __launch_bounds__(1024) void k_i8_long_rows(I8Quantize p) {
    __shared__ float tops[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r = blockIdx.x;
    int64_t lo = 0, hi = p.groups.rows;
    if (p.groups.offsets) {
        lo = min(max(p.groups.offsets[0], 0), p.groups.rows);
        hi = min(p.groups.offsets[p.groups.groups], p.groups.rows);
    }
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
    top = wave_max(top);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    top = 0.0f;
    for (int w = 0; w < 16; ++w) top = max_magnitude(top, tops[w], 0.0f);
    const float s = scale_of(top);
    const Scaled by[1] = {Scaled(s)};
    for (int c = (int)threadIdx.x * 8; c < (cols + 15) / 16 * 16; c += 1024 * 8) {
        float x[8];
        get(c, x);
        const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
        *reinterpret_cast<uint2 *>(p.q + r * p.ld + c) = make_uint2(quantize4(a, by), quantize4(b, by));
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

template <int TYPE>
__global__ __launch_bounds__(256) void k_i8_column_scales(I8Quantize p, int parts) {
    __shared__ float tops[4][kI8ColumnCols];
    I8Place at;
    if (!i8_find(p.groups, kI8ColumnRows, (uint32_t)parts, blockIdx.x, at)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int part = (int)(at.piece % (uint32_t)parts), r0 = at.span.lo + (int)(at.piece / (uint32_t)parts) * kI8ColumnRows;
    const int r1 = min(r0 + kI8ColumnRows, at.span.hi), cols = (int)p.cols, c = part * kI8ColumnCols + lane * 8;
    float top[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) top[i] = 0.0f;
    for (int r = r0 + wave; r < r1; r += 16) {                  // four rows at a time
        Eight<TYPE> in[4];
        int64_t from[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            from[u] = source_row(p, min(r + 4 * u, r1 - 1));    // (a row twice changes no maximum)
            in[u].load(static_cast<const typename Eight<TYPE>::T *>(p.X) + max(from[u], (int64_t)0) * p.ldx + c, cols - c, cols >= 8);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float x[8];
            in[u].move_down(from[u] < 0 ? 8 : Eight<TYPE>::down(cols - c, cols >= 8));
            in[u].get(x);
#pragma unroll
            for (int i = 0; i < 8; ++i) top[i] = max_magnitude(top[i], x[i], 0.0f);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) tops[wave][lane * 8 + i] = top[i];
    __syncthreads();
    for (int i = threadIdx.x; i < kI8ColumnCols; i += 256) {
        const float most = max_magnitude(max_magnitude(tops[0][i], tops[1][i], tops[2][i]), tops[3][i], 0.0f);
        if (part * kI8ColumnCols + i < cols)
            atomicMax(reinterpret_cast<uint32_t *>(p.scale_t + at.span.group * p.ld_scale_t + part * kI8ColumnCols + i), __builtin_bit_cast(uint32_t, scale_of(most)));
    }
}

// A tile of 128 x 128 of a group: thread (rg, cg) = (t / 16, t % 16) has rows 4 rg + i and columns 8 cg + j, and the bytes of a column change places in LDS, where
// the 16-byte chunk r / 16 of column c is at place (r / 16) ^ (c / 8 % 8).
template <int TYPE>
__global__ __launch_bounds__(kI8TileThreads) void k_i8_turn(I8Quantize p, int tiles_n) {
    __shared__ __align__(16) uint8_t turned[128 * 128];
    I8Place at;
    if (!i8_find(p.groups, 128, (uint32_t)tiles_n, blockIdx.x, at)) return;
    const int t = threadIdx.x, rg = t >> 4, cg = t & 15;
    const int tr = (int)(at.piece / (uint32_t)tiles_n), c0 = ((int)(at.piece % (uint32_t)tiles_n)) * 128;
    const int r0 = at.span.lo + tr * 128, rows = min(128, at.span.hi - r0), cols = (int)p.cols, c = c0 + 8 * cg;
    Eight<TYPE> in[4];
    int64_t from[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        from[i] = source_row(p, r0 + min(4 * rg + i, rows - 1));
        in[i].load(static_cast<const typename Eight<TYPE>::T *>(p.X) + max(from[i], (int64_t)0) * p.ldx + c, cols - c, cols >= 8);
    }
    const float *const scale = p.scale_t + at.span.group * p.ld_scale_t;
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        in[i].move_down(from[i] < 0 || 4 * rg + i >= rows ? 8 : Eight<TYPE>::down(cols - c, cols >= 8));
        in[i].get(x[i]);
    }
    uint8_t *const to = turned + 8 * cg * 128 + (rg / 4 ^ (cg & 7)) * 16 + rg % 4 * 4;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const Scaled by[1] = {Scaled(scale[min(c + j, cols - 1)])};
        const float column[4] = {x[0][j], x[1][j], x[2][j], x[3][j]};
        *reinterpret_cast<uint32_t *>(to + j * 128) = quantize4(column, by);
    }
    __syncthreads();
    const int64_t first = p.side_by_side ? i8_first_col(at.span) + tr * 128 : (int64_t)at.span.group * p.cols * p.ldt + tr * 128;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        const int row = pass * 64 + (t >> 3), chunk = t & 7;
        if (c0 + row < cols && (p.side_by_side || chunk * 16 < rows))
            *reinterpret_cast<f8_v4i *>(p.qt + first + (c0 + row) * p.ldt + chunk * 16) =
                *reinterpret_cast<const f8_v4i *>(turned + row * 128 + (chunk ^ (row >> 3 & 7)) * 16);
    }
}

template <int TYPE>
hipError_t launch(const I8Quantize &p, hipStream_t stream) {
    const int64_t rows = p.groups.rows, cols = p.cols;
    if (p.q) {
        const dim3 quarter((unsigned)((rows + 3) / 4)), whole((unsigned)rows), threads(kI8RowThreads);
        if (cols <= 512) hipLaunchKernelGGL((k_i8_rows<TYPE, 1, true>), quarter, threads, 0, stream, p);
        else if (cols <= 2048) hipLaunchKernelGGL((k_i8_rows<TYPE, 1, false>), whole, threads, 0, stream, p);
        else if (cols <= 4096) hipLaunchKernelGGL((k_i8_rows<TYPE, 2, false>), whole, threads, 0, stream, p);
        else if (cols <= 8192) hipLaunchKernelGGL((k_i8_rows<TYPE, 4, false>), whole, threads, 0, stream, p);
        else if (cols <= kI8MostHeld) hipLaunchKernelGGL((k_i8_rows<TYPE, 8, false>), whole, threads, 0, stream, p);
        else hipLaunchKernelGGL((k_i8_long_rows<TYPE>), whole, dim3(1024), 0, stream, p);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (!p.qt) return hipSuccess;
    const int groups = p.groups.groups;
    const int64_t run = p.side_by_side ? cols : groups * cols;  // of scales without a gap
    hipLaunchKernelGGL(k_i8_least_scales, dim3((unsigned)f8_ceil(run, 256), p.side_by_side ? (unsigned)groups : 1u), dim3(256), 0, stream, p.scale_t, p.ld_scale_t, (int)run);
    if (hipError_t e = hipGetLastError()) return e;
    const int64_t parts = f8_ceil(cols, kI8ColumnCols), tiles = f8_ceil(cols, 128);
    const auto units = [&](int64_t each) { return i8_quantize_units(p.groups, each); };
    hipLaunchKernelGGL((k_i8_column_scales<TYPE>), dim3((unsigned)(f8_ceil(units(kI8ColumnRows) * parts, 8) * 8)), dim3(256), 0, stream, p, (int)parts);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL((k_i8_turn<TYPE>), dim3((unsigned)(f8_ceil(units(128) * tiles, 8) * 8)), dim3(kI8TileThreads), 0, stream, p, (int)tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_i8_quantize(const I8Quantize &args, int type, hipStream_t stream) {
    return type == kF8Bf16 ? launch<kF8Bf16>(args, stream) : type == kF8F16 ? launch<kF8F16>(args, stream) : launch<kF8F32>(args, stream);
}

}  // namespace oz2
