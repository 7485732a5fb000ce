// Numbers to E4M3 with a power of two per block: the smallest 2^s, s >= -126, with max|x| <= 448 2^s over the finite numbers of the block,
// 2^0 for none or zeros only.  x 2^-s is exact, so the rounding to E4M3 (to nearest even, by the conversion instruction) is the
// only one; NaN and infinities become NaN.  448 = 1.75 2^8: with max = f 2^e, 1 <= f < 2, s = e - 8 for f <= 1.75, else e - 7, which
// are integer operations on the bits.
//
// A block of one row for the matrix as it is and for its transpose, or of 128 x 128 for both, come from one read: a workgroup
// holds a tile of 128 x 128 in registers, 8 x 8 numbers per thread, and turns the bytes of the transpose through LDS.
// Bound: HBM; the smallest calls by latency.
#include "oz2_f8_device.hpp"

namespace oz2 {
namespace {

__device__ __forceinline__ float finite_magnitude(float x) {
    const float a = __builtin_fabsf(x);
    return a < __builtin_inff() ? a : 0.0f;                    // also false for NaN
}
// The scale of a block as the byte of E8M0, and 2^-s.
__device__ __forceinline__ int scale_byte(float top) {
    const int bits = __builtin_bit_cast(int, top);
    return bits ? max((bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0), 1) : 127;
}
__device__ __forceinline__ float inverse_scale(int byte) { return __builtin_bit_cast(float, (254 - byte) << 23); }

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// 8 numbers of a row from X[at] on, of which `valid` exist (zeros for the others); vec: 8 at once may be loaded.
template <int TYPE>
__device__ __forceinline__ void load8(const void *X, int64_t at, int valid, bool vec, float (&x)[8]) {
    typedef F8Number<TYPE> N;
    const typename N::T *const from = static_cast<const typename N::T *>(X) + at;
    if (vec && valid >= 8) {
        if constexpr (TYPE == kF8F32) {
            const f8_v4f lo = reinterpret_cast<const f8_v4f *>(from)[0], hi = reinterpret_cast<const f8_v4f *>(from)[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = lo[i]; x[4 + i] = hi[i]; }
        } else {
            const f8_v4i w = *reinterpret_cast<const f8_v4i *>(from);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = N::get((uint16_t)((uint32_t)w[i / 2] >> (i % 2 * 16)));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < valid ? N::get(from[i]) : 0.0f;
}

constexpr int kTurnLd = 128 + 16;                              // bytes of a column of the tile in LDS

struct TileLds {
    float top[4][128];
    uint8_t turn[128 * kTurnLd];
};

// A tile of 128 x 128 in registers: thread (rg, cg) = (t / 16, t % 16) has rows 8 rg + i and columns 8 cg + j.  rows, cols: those of the
// tile that exist (bytes are written for whole chunks of 16 of which one does).  r0, c0: its place in the matrix; SQUARE: one
// scale for the tile.
template <bool SQUARE>
__device__ __forceinline__ void write_tile(const float (&x)[8][8], TileLds &lds, int64_t r0, int64_t c0, int rows, int cols, const F8Target &as_is,
                                           const F8Target &transposed) {
    const int t = threadIdx.x, rg = t >> 4, cg = t & 15, wave = t >> 6;
    float row_top[8], col_top[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) row_top[i] = col_top[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float a = finite_magnitude(x[i][j]);
            row_top[i] = fmaxf(row_top[i], a);
            if (!SQUARE) col_top[j] = fmaxf(col_top[j], a);
        }
    int all = 127;                                             // the byte of the square block
    if (SQUARE) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, row_top[i]);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        if ((t & 63) == 0) lds.top[wave][0] = top;
        __syncthreads();
        all = scale_byte(fmaxf(fmaxf(lds.top[0][0], lds.top[1][0]), fmaxf(lds.top[2][0], lds.top[3][0])));
    }
    if (as_is.q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 8 * rg + i;
            int byte = all;
            if (!SQUARE) {
                float top = row_top[i];
#pragma unroll
                for (int d = 1; d < 16; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
                byte = scale_byte(top);
            }
            const float inv = inverse_scale(byte);
            if (r < rows && (8 * cg & ~15) < cols)
                *reinterpret_cast<uint2 *>(as_is.q + (r0 + r) * as_is.ld + c0 + 8 * cg) =
                    make_uint2(pack4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv), pack4(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv));
            if (!SQUARE && cg == 0 && r < rows) as_is.scale[(r0 + r) * as_is.ld_scale + c0 / 128] = (uint8_t)byte;
        }
        if (SQUARE && t == 0) as_is.scale[r0 / 128 * as_is.ld_scale + c0 / 128] = (uint8_t)all;
    }
    if (transposed.q) {
        if (!SQUARE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float top = col_top[j];
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                if ((t & 63) < 16) lds.top[wave][8 * cg + j] = top;
            }
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = 8 * cg + j;
            const int byte = SQUARE ? all : scale_byte(fmaxf(fmaxf(lds.top[0][c], lds.top[1][c]), fmaxf(lds.top[2][c], lds.top[3][c])));
            const float inv = inverse_scale(byte);
            *reinterpret_cast<uint2 *>(lds.turn + c * kTurnLd + 8 * rg) =
                make_uint2(pack4(x[0][j] * inv, x[1][j] * inv, x[2][j] * inv, x[3][j] * inv), pack4(x[4][j] * inv, x[5][j] * inv, x[6][j] * inv, x[7][j] * inv));
            if (!SQUARE && rg == 0 && c < cols) transposed.scale[(c0 + c) * transposed.ld_scale + r0 / 128] = (uint8_t)byte;
        }
        if (SQUARE && t == 0) transposed.scale[c0 / 128 * transposed.ld_scale + r0 / 128] = (uint8_t)all;
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < 4; ++pass) {
            const int c = pass * 32 + (t >> 3), chunk = t & 7;
            if (c < cols && chunk * 16 < rows)
                *reinterpret_cast<f8_v4i *>(transposed.q + (c0 + c) * transposed.ld + r0 + chunk * 16) = *reinterpret_cast<const f8_v4i *>(lds.turn + c * kTurnLd + chunk * 16);
        }
    }
}

template <int TYPE, bool SQUARE>
__global__ __launch_bounds__(256) void k_f8_quantize_tiles(const void *X, int64_t rows, int64_t cols, int64_t ldx, int tiles_n, Divisor by_row, bool vec,
                                                           F8Target as_is, F8Target transposed) {
    __shared__ __align__(16) TileLds lds;
    const int tr = divide((int)blockIdx.x, by_row), tc = (int)blockIdx.x - tr * tiles_n;
    const int64_t r0 = (int64_t)tr * 128, c0 = (int64_t)tc * 128;
    const int rg = threadIdx.x >> 4, cg = threadIdx.x & 15;
    const int here_r = (int)(rows - r0 < 128 ? rows - r0 : 128), here_c = (int)(cols - c0 < 128 ? cols - c0 : 128);
    float x[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) load8<TYPE>(X, (r0 + 8 * rg + i) * ldx + c0 + 8 * cg, 8 * rg + i < here_r ? here_c - 8 * cg : 0, vec, x[i]);
    write_tile<SQUARE>(x, lds, r0, c0, here_r, here_c, as_is, transposed);
}

// Blocks of one row, as they are: 16 lanes take a block, 8 numbers each.
template <int TYPE>
__global__ __launch_bounds__(256) void k_f8_quantize_rows(const void *X, int64_t rows, int64_t cols, int64_t ldx, int blocks, Divisor by_row, bool vec, F8Target out) {
    const int unit = (int)blockIdx.x * 16 + (threadIdx.x >> 4), cg = threadIdx.x & 15;
    const int r = divide(unit, by_row), b = unit - r * blocks;
    if (r >= rows) return;
    const int here = (int)(cols - (int64_t)b * 128 < 128 ? cols - (int64_t)b * 128 : 128);
    float x[8], top = 0.0f;
    load8<TYPE>(X, r * ldx + (int64_t)b * 128 + 8 * cg, here - 8 * cg, vec, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, finite_magnitude(x[j]));
#pragma unroll
    for (int d = 1; d < 16; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const int byte = scale_byte(top);
    const float inv = inverse_scale(byte);
    if ((8 * cg & ~15) < here)
        *reinterpret_cast<uint2 *>(out.q + r * out.ld + (int64_t)b * 128 + 8 * cg) =
            make_uint2(pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), pack4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
    if (cg == 0) out.scale[r * out.ld_scale + b] = (uint8_t)byte;
}

// dZ = (dH up act'(gate), dH act(gate)) of the gated block, in 8 bits with blocks of one row, as it is and transposed, without its
// ever being written in full.  The columns between f and `up` are zeros.
template <int TYPE>
__global__ __launch_bounds__(256) void k_f8_gated_grad(const void *Z, int64_t ldz, const void *dH, int64_t ldh, int64_t m, int64_t f, int64_t up, int act,
                                                       int tiles_n, Divisor by_row, bool z_vec, bool h_vec, F8Target D, F8Target DT) {
    __shared__ __align__(16) TileLds lds;
    const int tr = divide((int)blockIdx.x, by_row), tc = (int)blockIdx.x - tr * tiles_n;
    const int64_t r0 = (int64_t)tr * 128, c0 = (int64_t)tc * 128;
    const int rg = threadIdx.x >> 4, cg = threadIdx.x & 15;
    const int here_r = (int)(m - r0 < 128 ? m - r0 : 128), here_c = (int)(f - c0 < 128 ? f - c0 : 128);
    float dg[8][8], du[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int valid = 8 * rg + i < here_r ? here_c - 8 * cg : 0;
        const int64_t r = r0 + 8 * rg + i, c = c0 + 8 * cg;
        float g[8], u[8], h[8];
        load8<TYPE>(Z, r * ldz + c, valid, z_vec, g);
        load8<TYPE>(Z, r * ldz + up + c, valid, z_vec, u);
        load8<TYPE>(dH, r * ldh + c, valid, h_vec, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float p = f8_gate(g[j], act);
            dg[i][j] = h[j] * u[j] * f8_slope(g[j], p, act);
            du[i][j] = h[j] * (g[j] * p);
        }
    }
    write_tile<false>(dg, lds, r0, c0, here_r, 128, D, DT);
    __syncthreads();
    write_tile<false>(du, lds, r0, up + c0, here_r, here_c, D, DT);
}

// Rows of 8 numbers at columns that are multiples of 8 may be loaded 16 bytes at a time.
bool vec_rows(const void *X, int64_t ld, int type) {
    return reinterpret_cast<uintptr_t>(X) % 16 == 0 && ld * f8_type_bytes(type) % 16 == 0;
}

template <int TYPE>
hipError_t launch_quantize(const void *X, int64_t rows, int64_t cols, int64_t ldx, bool square, const F8Target &as_is, const F8Target &transposed,
                           hipStream_t stream) {
    const int tiles_m = (int)((rows + 127) / 128), tiles_n = (int)((cols + 127) / 128);
    const bool vec = vec_rows(X, ldx, TYPE);
    if (!square && !transposed.q) {
        const int64_t units = rows * tiles_n;
        hipLaunchKernelGGL((k_f8_quantize_rows<TYPE>), dim3((unsigned)((units + 15) / 16)), dim3(256), 0, stream, X, rows, cols, ldx, tiles_n, make_divisor(tiles_n), vec, as_is);
    } else if (square) {
        hipLaunchKernelGGL((k_f8_quantize_tiles<TYPE, true>), dim3((unsigned)(tiles_m * tiles_n)), dim3(256), 0, stream, X, rows, cols, ldx, tiles_n, make_divisor(tiles_n), vec, as_is, transposed);
    } else {
        hipLaunchKernelGGL((k_f8_quantize_tiles<TYPE, false>), dim3((unsigned)(tiles_m * tiles_n)), dim3(256), 0, stream, X, rows, cols, ldx, tiles_n, make_divisor(tiles_n), vec, as_is, transposed);
    }
    return hipGetLastError();
}

template <int TYPE>
hipError_t launch_grad(const void *Z, int64_t ldz, const void *dH, int64_t ldh, int64_t m, int64_t f, int64_t up, int act, const F8Target &D,
                       const F8Target &DT, hipStream_t stream) {
    const int tiles_m = (int)((m + 127) / 128), tiles_n = (int)((f + 127) / 128);
    hipLaunchKernelGGL((k_f8_gated_grad<TYPE>), dim3((unsigned)(tiles_m * tiles_n)), dim3(256), 0, stream, Z, ldz, dH, ldh, m, f, up, act, tiles_n,
                       make_divisor(tiles_n), vec_rows(Z, ldz, TYPE), vec_rows(dH, ldh, TYPE), D, DT);
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
