// Numbers to E4M3 with a power of two per block: the smallest 2^s, s >= -126, with max|x| <= 448 2^s over the finite numbers of the block,
// 2^0 for none or zeros only.  x 2^-s is exact, so the rounding to E4M3 (to nearest even, by the conversion instruction) is the
// only one; NaN and infinities become NaN.  448 = 1.75 2^8: with max = f 2^e, 1 <= f < 2, s = e - 8 for f <= 1.75, else e - 7, which
// are integer operations on the bits.
//
// A block of one row for the matrix as it is and for its transpose, or of 128 x 128 for both, come from one read: a workgroup
// holds a tile of 128 x 128 in registers, 4 x 8 numbers per thread, and turns the bytes of the transpose through LDS.
// 16384 x 8192 bf16 in blocks of 128 x 128, as it is and transposed: 111 to 113 us, 4.7 to 4.8 TB/s; as it is only, by rows, 71 to 79 us, 5.1 to 5.7 TB/s; 1500 x 1111 f32
// 5.8 us, 64 x 8192 2.9 us.  Bound: HBM; the smallest calls by latency.
#include "oz2_f8_device.hpp"

namespace oz2 {
namespace {

// The largest of top, |x| and |y| in one instruction, NaN if one of them is.  (v_max3_f32 passes over NaN, and having met a signalling one it
// has forgotten what came before.)  Whatever is not below infinity at the end has met NaN or an infinity, and then the maxima are taken
// again with finite_magnitude.
__device__ __forceinline__ float max_magnitude(float top, float x, float y) {
    float r;
    asm("v_maximum3_f32 %0, %1, |%2|, |%3|" : "=v"(r) : "v"(top), "v"(x), "v"(y));
    return r;
}
__device__ __forceinline__ float finite_magnitude(float x) {
    const float a = __builtin_fabsf(x);
    return a < __builtin_inff() ? a : 0.0f;                    // also false for NaN
}
__device__ __forceinline__ bool is_finite(float top) { return top < __builtin_inff(); }

// Magnitudes by their bits, which are in the same order and need no care for NaN.
// The maximum over the 16 lanes of a row of lanes, in all of them (rotations within the row, part of the instruction).
template <int BY>
__device__ __forceinline__ uint32_t max_rotated(uint32_t x) {
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + BY, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t max_of_16(float x) {
    return max_rotated<8>(max_rotated<4>(max_rotated<2>(max_rotated<1>(__builtin_bit_cast(uint32_t, x)))));
}
// The maxima of x over the lanes l and l + 32 where l < 32, of y where l >= 32; the same for l, l + 16 in the even and odd quarters.
__device__ __forceinline__ uint32_t max_of_halves(uint32_t x, uint32_t y) {
    const auto s = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    return max((uint32_t)s[0], (uint32_t)s[1]);
}
__device__ __forceinline__ uint32_t max_of_quarters(uint32_t x, uint32_t y) {
    const auto s = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    return max((uint32_t)s[0], (uint32_t)s[1]);
}

// The scale of a block as the byte of E8M0, and 2^-s.
__device__ __forceinline__ int scale_byte(uint32_t top) {
    const int bits = (int)top;
    return bits ? max((bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0), 1) : 127;
}
__device__ __forceinline__ float inverse_scale(int byte) { return __builtin_bit_cast(float, (254 - byte) << 23); }

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// 8 numbers of a row as they lie in memory, of which `valid` exist (zeros for the others), and in binary32.
template <int TYPE>
struct Eight {
    static constexpr int kWords = TYPE == kF8F32 ? 2 : 1;
    f8_v4i w[kWords];
    typedef typename F8Number<TYPE>::T T;
    __device__ __forceinline__ void load(const T *from) { __builtin_memcpy(w, from, sizeof w); }
    // Of a row that ends at from[valid - 1] (`valid` may be negative), to be followed by move_down(down(valid, eight)).  A row of 8 or more numbers
    // (`eight`) is read as its last 8, which are then moved down; number by number, one wait after the other, tiles at the edge took as
    // long as all others (as they are, 16384 x 8191: 105 us instead of 78; the gradient's, 8192 x 8191, 256 instead of 164).
    __device__ __forceinline__ void load(const T *from, int valid, bool eight) {
        if (eight) {
            load(from - max(8 - valid, 0));
            return;
        }
        uint32_t words[4 * kWords];
#pragma unroll
        for (int i = 0; i < 4 * kWords; ++i) words[i] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) {
                if constexpr (TYPE == kF8F32) words[i] = __builtin_bit_cast(uint32_t, from[i]);
                else words[i / 2] |= (uint32_t)from[i] << (i % 2 * 16);
            }
#pragma unroll
        for (int i = 0; i < 4 * kWords; ++i) w[i / 4][i % 4] = (int)words[i];
    }
    static __device__ __forceinline__ int down(int valid, bool eight) { return eight ? min(max(8 - valid, 0), 8) : 0; }
    __device__ __forceinline__ void move_down(int by) {        // by 0 to 8 numbers, zeros following
        constexpr int N = 4 * kWords;
        uint32_t words[N];
#pragma unroll
        for (int i = 0; i < N; ++i) words[i] = (uint32_t)w[i / 4][i % 4];
#pragma unroll
        for (int step = 1; step <= 8; step *= 2) {
            const bool move = by & step;
            const int whole = step * N / 8;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t next = i + max(whole, 1) < N ? words[i + max(whole, 1)] : 0;
                words[i] = !move ? words[i] : whole ? next : __builtin_amdgcn_alignbyte(next, words[i], 2);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) w[i / 4][i % 4] = (int)words[i];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (TYPE == kF8F32) {
                const int word = w[i / 4][i % 4];
                x[i] = __builtin_bit_cast(float, word);
            } else x[i] = F8Number<TYPE>::get((uint16_t)((uint32_t)w[0][i / 2] >> (i % 2 * 16)));
        }
    }
};

constexpr int kTileThreads = kF8TileThreads, kTileWaves = kTileThreads / 64;
constexpr int kOwn = 128 * 16 / kTileThreads;                  // rows of a thread

// The rows of a thread of a tile, which has `rows` rows and `cols` columns; X at the tile's first number, with `before` more in front of it in its row.
// settle_rows comes when all that a thread reads has been asked for: what it does at the edges waits for the numbers.
template <int TYPE>
__device__ __forceinline__ void load_rows(Eight<TYPE> (&in)[kOwn], const void *X, int64_t at, int64_t ld, int rows, int cols, int64_t before) {
    const int rg = threadIdx.x >> 4, cg = threadIdx.x & 15;
    const typename Eight<TYPE>::T *const from = static_cast<const typename Eight<TYPE>::T *>(X) + at + 8 * cg;
    if (rows == 128 && cols == 128) {                          // uniform
#pragma unroll
        for (int i = 0; i < kOwn; ++i) in[i].load(from + (kOwn * rg + i) * ld);
    } else {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) in[i].load(from + min(kOwn * rg + i, rows - 1) * ld, cols - 8 * cg, before + cols >= 8);
    }
}
template <int TYPE>
__device__ __forceinline__ void settle_rows(Eight<TYPE> (&in)[kOwn], int rows, int cols, int64_t before) {
    if (rows == 128 && cols == 128) return;
    const int rg = threadIdx.x >> 4, cg = threadIdx.x & 15;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) in[i].move_down(kOwn * rg + i < rows ? Eight<TYPE>::down(cols - 8 * cg, before + cols >= 8) : 8);
}

struct __align__(16) TileLds {
    uint32_t top[kTileWaves][128];                             // bits of magnitudes
    uint8_t turn[128 * 128];                                   // the transpose: 16-byte chunk r / 16 of column c is at place (r / 16) ^ (c / 8 % 8)
};

// A tile of 128 x 128 in registers: thread (rg, cg) = (t / 16, t % 16) has rows kOwn rg + i and columns 8 cg + j.  rows, cols: those of the
// tile that exist (bytes are written for whole chunks of 16 of which one does), all of them if WHOLE.  r0, c0: its place in the matrix;
// SQUARE: one scale for the tile.
template <bool SQUARE, bool WHOLE>
__device__ __forceinline__ void write_tile(const float (&x)[kOwn][8], TileLds &lds, int64_t r0, int64_t c0, int rows, int cols, const F8Target &as_is,
                                           const F8Target &transposed) {
    const int t = threadIdx.x, rg = t >> 4, cg = t & 15, wave = t >> 6;
    float row_top[kOwn], col_top[8];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        row_top[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; j += 2) row_top[i] = max_magnitude(row_top[i], x[i][j], x[i][j + 1]);
    }
    if (!SQUARE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            col_top[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < kOwn; i += 2) col_top[j] = max_magnitude(col_top[j], x[i][j], x[i + 1][j]);
        }
    }
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < kOwn; i += 2) top = max_magnitude(top, row_top[i], row_top[i + 1]);
    if (__builtin_expect(__any(!is_finite(top)), 0)) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) row_top[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) col_top[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = x[i][j];
                asm volatile("" : "+v"(v));                    // (or all this is computed beforehand, needed or not)
                const float a = finite_magnitude(v);
                row_top[i] = fmaxf(row_top[i], a);
                if (!SQUARE) col_top[j] = fmaxf(col_top[j], a);
            }
        top = 0.0f;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) top = fmaxf(top, row_top[i]);
    }
    float inv_all = 1.0f;                                      // of the square block
    if (SQUARE) {
        uint32_t most = max_of_16(top);
        most = max_of_quarters(most, most);
        most = max_of_halves(most, most);
        if ((t & 63) == 0) lds.top[wave][0] = most;
        __syncthreads();
        most = lds.top[0][0];
#pragma unroll
        for (int v = 1; v < kTileWaves; ++v) most = max(most, lds.top[v][0]);
        const int byte = scale_byte(most);
        inv_all = inverse_scale(byte);
        if (t == 0) {
            if (as_is.q) as_is.scale[r0 / 128 * as_is.ld_scale + c0 / 128] = (uint8_t)byte;
            if (transposed.q) transposed.scale[c0 / 128 * transposed.ld_scale + r0 / 128] = (uint8_t)byte;
        }
    }
    if (!SQUARE && transposed.q) {
        // Columns j, j + 4 by halves of the wavefront, then j, j + 2 by its quarters: a lane is left with columns jq and jq + 1.
        const int jq = (t >> 5 & 1) * 4 + (t >> 4 & 1) * 2;
        uint32_t half[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) half[j] = max_of_halves(__builtin_bit_cast(uint32_t, col_top[j]), __builtin_bit_cast(uint32_t, col_top[j + 4]));
        *reinterpret_cast<uint2 *>(&lds.top[wave][8 * cg + jq]) = make_uint2(max_of_quarters(half[0], half[2]), max_of_quarters(half[1], half[3]));
    }
    if (as_is.q) {
        uint8_t *to = as_is.q + (r0 + kOwn * rg) * as_is.ld + c0 + 8 * cg, *scale = as_is.scale + (r0 + kOwn * rg) * as_is.ld_scale + c0 / 128;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int byte = SQUARE ? 0 : scale_byte(max_of_16(row_top[i]));
            const float inv = SQUARE ? inv_all : inverse_scale(byte);
            const uint2 packed = make_uint2(pack4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv),
                                            pack4(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv));
            if (WHOLE || (kOwn * rg + i < rows && (8 * cg & ~15) < cols)) *reinterpret_cast<uint2 *>(to) = packed;
            if (!SQUARE && cg == 0 && (WHOLE || kOwn * rg + i < rows)) *scale = (uint8_t)byte;
            to += as_is.ld;
            scale += as_is.ld_scale;
        }
    }
    if (transposed.q) {
        f8_v4f inv[2] = {{inv_all, inv_all, inv_all, inv_all}, {inv_all, inv_all, inv_all, inv_all}};
        if (!SQUARE) {
            __syncthreads();
            if (t < 128) {                                     // (a thread reads and writes its own column)
                uint32_t most = lds.top[0][t];
#pragma unroll
                for (int v = 1; v < kTileWaves; ++v) most = max(most, lds.top[v][t]);
                const int byte = scale_byte(most);
                if (WHOLE || t < cols) transposed.scale[(c0 + t) * transposed.ld_scale + r0 / 128] = (uint8_t)byte;
                lds.top[0][t] = (uint32_t)(254 - byte) << 23;  // inverse_scale's bits
            }
            __syncthreads();
            inv[0] = *reinterpret_cast<const f8_v4f *>(&lds.top[0][8 * cg]);
            inv[1] = *reinterpret_cast<const f8_v4f *>(&lds.top[0][8 * cg + 4]);
        }
        uint8_t *const turn = lds.turn + 8 * cg * 128 + (rg / 4 ^ (cg & 7)) * 16 + rg % 4 * 4;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = inv[j / 4][j % 4];
            *reinterpret_cast<uint32_t *>(turn + j * 128) = pack4(x[0][j] * v, x[1][j] * v, x[2][j] * v, x[3][j] * v);
        }
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < 1024 / kTileThreads; ++pass) {
            const int c = pass * (kTileThreads / 8) + (t >> 3), chunk = t & 7;
            if (WHOLE || (c < cols && chunk * 16 < rows))
                *reinterpret_cast<f8_v4i *>(transposed.q + (c0 + c) * transposed.ld + r0 + chunk * 16) =
                    *reinterpret_cast<const f8_v4i *>(lds.turn + c * 128 + (chunk ^ (c >> 3 & 7)) * 16);
        }
    }
}

template <int TYPE, bool SQUARE>
__global__ __launch_bounds__(kTileThreads) void k_f8_quantize_tiles(const void *X, int64_t rows, int64_t cols, int64_t ldx, int tiles_n, Divisor by_row,
                                                           F8Target as_is, F8Target transposed) {
    __shared__ __align__(16) TileLds lds;
    const int tr = divide((int)blockIdx.x, by_row), tc = (int)blockIdx.x - tr * tiles_n;
    const int64_t r0 = (int64_t)tr * 128, c0 = (int64_t)tc * 128;
    const int here_r = (int)(rows - r0 < 128 ? rows - r0 : 128), here_c = (int)(cols - c0 < 128 ? cols - c0 : 128);
    Eight<TYPE> in[kOwn];
    load_rows<TYPE>(in, X, r0 * ldx + c0, ldx, here_r, here_c, c0);
    settle_rows<TYPE>(in, here_r, here_c, c0);
    float x[kOwn][8];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) in[i].get(x[i]);
    if (here_r == 128 && here_c == 128) write_tile<SQUARE, true>(x, lds, r0, c0, here_r, here_c, as_is, transposed);
    else write_tile<SQUARE, false>(x, lds, r0, c0, here_r, here_c, as_is, transposed);
}

// Blocks of one row, as they are: 16 lanes take a block, 8 numbers each.
template <int TYPE>
__global__ __launch_bounds__(kF8RowThreads) void k_f8_quantize_rows(const void *X, int64_t rows, int64_t cols, int64_t ldx, int blocks, Divisor by_row, F8Target out) {
    const int unit = (int)blockIdx.x * 16 + (threadIdx.x >> 4), cg = threadIdx.x & 15;
    const int r = divide(unit, by_row), b = unit - r * blocks;
    if (r >= rows) return;
    const int here = (int)(cols - (int64_t)b * 128 < 128 ? cols - (int64_t)b * 128 : 128);
    float x[8], top = 0.0f;
    Eight<TYPE> in;
    in.load(static_cast<const typename Eight<TYPE>::T *>(X) + r * ldx + (int64_t)b * 128 + 8 * cg, here - 8 * cg, cols >= 8);
    in.move_down(Eight<TYPE>::down(here - 8 * cg, cols >= 8));
    in.get(x);
#pragma unroll
    for (int j = 0; j < 8; j += 2) top = max_magnitude(top, x[j], x[j + 1]);
    if (__any(!is_finite(top))) {
        top = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v = x[j];
            asm volatile("" : "+v"(v));
            top = fmaxf(top, finite_magnitude(v));
        }
    }
    const int byte = scale_byte(max_of_16(top));
    const float inv = inverse_scale(byte);
    if ((8 * cg & ~15) < here)
        *reinterpret_cast<uint2 *>(out.q + r * out.ld + (int64_t)b * 128 + 8 * cg) =
            make_uint2(pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), pack4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
    if (cg == 0) out.scale[r * out.ld_scale + b] = (uint8_t)byte;
}

// dZ = (dH up act'(gate), dH act(gate)) of the gated block, in 8 bits with blocks of one row, as it is and transposed, without its
// ever being written in full.  The columns between f and `up` are zeros.  A workgroup takes a tile of one of the two parts (both at
// once had no room in registers: 226 us and more at 8192 x 8192 instead of 150); the other part's, 8 ids further, finds what
// both read in the same L2.
template <int TYPE>
__global__ __launch_bounds__(kTileThreads, 4) void k_f8_gated_grad(const void *Z, int64_t ldz, const void *dH, int64_t ldh, int64_t m, int64_t f, int64_t up,
                                                                   int act, int tiles, int tiles_n, Divisor by_row, F8Target D, F8Target DT) {
    __shared__ TileLds lds;
    const int tile = (int)(blockIdx.x >> 4 << 3 | (blockIdx.x & 7)), part = (int)(blockIdx.x >> 3 & 1);
    if (tile >= tiles) return;
    const int tr = divide(tile, by_row), tc = tile - tr * tiles_n;
    const int64_t r0 = (int64_t)tr * 128, c0 = (int64_t)tc * 128;
    const int here_r = (int)(m - r0 < 128 ? m - r0 : 128), here_c = (int)(f - c0 < 128 ? f - c0 : 128);
    Eight<TYPE> gate[kOwn], lift[kOwn], grad[kOwn];
    load_rows<TYPE>(gate, Z, r0 * ldz + c0, ldz, here_r, here_c, c0);
    if (!part) load_rows<TYPE>(lift, Z, r0 * ldz + up + c0, ldz, here_r, here_c, c0);
    load_rows<TYPE>(grad, dH, r0 * ldh + c0, ldh, here_r, here_c, c0);
    settle_rows<TYPE>(gate, here_r, here_c, c0);
    if (!part) settle_rows<TYPE>(lift, here_r, here_c, c0);
    settle_rows<TYPE>(grad, here_r, here_c, c0);
    float x[kOwn][8];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        float g[8], h[8];
        gate[i].get(g);
        grad[i].get(h);
        if (part) {
            if (act) f8_times_act<1>(g, h, x[i]);
            else f8_times_act<0>(g, h, x[i]);
        } else {
            float u[8];
            lift[i].get(u);
            if (act) f8_times_slope<1>(g, u, h, x[i]);
            else f8_times_slope<0>(g, u, h, x[i]);
        }
    }
    const int64_t at = c0 + (part ? up : 0);
    const int cols = part ? here_c : 128;                      // (the columns between the parts are the first one's)
    if (here_r == 128 && cols == 128) write_tile<false, true>(x, lds, r0, at, here_r, cols, D, DT);
    else write_tile<false, false>(x, lds, r0, at, here_r, cols, D, DT);
}

template <int TYPE>
hipError_t launch_quantize(const void *X, int64_t rows, int64_t cols, int64_t ldx, bool square, const F8Target &as_is, const F8Target &transposed,
                           hipStream_t stream) {
    const int tiles_n = (int)f8_blocks(cols);
    const dim3 tiles((unsigned)f8_tile_groups(rows, cols));
    if (f8_by_rows(rows, cols, square, transposed.q != nullptr)) {
        hipLaunchKernelGGL((k_f8_quantize_rows<TYPE>), dim3((unsigned)f8_row_groups(rows, cols)), dim3(kF8RowThreads), 0, stream, X, rows, cols, ldx, tiles_n, make_divisor(tiles_n), as_is);
    } else if (square) {
        hipLaunchKernelGGL((k_f8_quantize_tiles<TYPE, true>), tiles, dim3(kTileThreads), 0, stream, X, rows, cols, ldx, tiles_n, make_divisor(tiles_n), as_is, transposed);
    } else {
        hipLaunchKernelGGL((k_f8_quantize_tiles<TYPE, false>), tiles, dim3(kTileThreads), 0, stream, X, rows, cols, ldx, tiles_n, make_divisor(tiles_n), as_is, transposed);
    }
    return hipGetLastError();
}

template <int TYPE>
hipError_t launch_grad(const void *Z, int64_t ldz, const void *dH, int64_t ldh, int64_t m, int64_t f, int64_t up, int act, const F8Target &D,
                       const F8Target &DT, hipStream_t stream) {
    const int tiles_n = (int)f8_blocks(f), tiles = (int)f8_tile_groups(m, f);
    hipLaunchKernelGGL((k_f8_gated_grad<TYPE>), dim3((unsigned)f8_grad_groups(m, f)), dim3(kTileThreads), 0, stream, Z, ldz, dH, ldh, m, f, up, act, tiles, tiles_n,
                       make_divisor(tiles_n), D, DT);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_quantize(const void *X, int type, int64_t rows, int64_t cols, int64_t ldx, bool square, const F8Target &as_is,
                              const F8Target &transposed, hipStream_t stream) {
    return type == kF8Bf16 ? launch_quantize<kF8Bf16>(X, rows, cols, ldx, square, as_is, transposed, stream)
         : type == kF8F16  ? launch_quantize<kF8F16>(X, rows, cols, ldx, square, as_is, transposed, stream)
                           : launch_quantize<kF8F32>(X, rows, cols, ldx, square, as_is, transposed, stream);
}

hipError_t launch_f8_gated_grad(const void *Z, int64_t ldz, const void *dH, int64_t ldh, int type, int64_t m, int64_t f, int64_t up,
                                int act, const F8Target &D, const F8Target &DT, hipStream_t stream) {
    return type == kF8Bf16 ? launch_grad<kF8Bf16>(Z, ldz, dH, ldh, m, f, up, act, D, DT, stream)
         : type == kF8F16  ? launch_grad<kF8F16>(Z, ldz, dH, ldh, m, f, up, act, D, DT, stream)
                           : launch_grad<kF8F32>(Z, ldz, dH, ldh, m, f, up, act, D, DT, stream);
}

}  // namespace oz2
