// Products of 8-bit integers with few rows of A (tokens that are decoded), alone or by group: every element of B is read once, straight into the registers of
// the matrix instruction, and C has no other work.  A workgroup takes 16 columns of C (of one group), its wavefronts take groups of 4 blocks of
// 128 of k in turn and add their sums through LDS.  A group with more than 16 MT rows is taken in parts, for which its columns of B are read again.
//
// 1 x 8192 x 8192 13.9 us, 4.8 TB/s; 8 rows of 64 experts, 4096 x 2048 each, 13.9 us, 4.8 TB/s (64 x 64 tiles: 15.5).  Bound: HBM (the bytes of B).
#include "oz2_i8_device.hpp"

namespace oz2 {
namespace {

constexpr int kWaves = 8;                                     // of a workgroup at most

// MT blocks of 16 rows of A.
template <int MT, I8Mode MODE>
__global__ __launch_bounds__(kWaves * 64) void k_i8_thin(I8Args p) {
    extern __shared__ f8_v4i sums[];                          // [wavefronts][MT][64]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = (int)blockDim.x >> 6;
    const int lrow = lane & 15, quarter = lane >> 4;
    int col0 = (int)blockIdx.x * 16, lo = 0, hi = p.m, group = 0;
    if constexpr (MODE == I8Mode::kRows) {
        const uint32_t parts = (uint32_t)(p.n + 15) / 16;
        I8Place at;
        if (!i8_find(p.groups, 1 << 30, parts, blockIdx.x, at)) return;   // (a unit is a group that has rows)
        col0 = (int)at.piece * 16;
        lo = at.span.lo;
        hi = at.span.hi;
        group = at.span.group;
    }
    const int KB = (p.k + kI8Block - 1) / kI8Block, whole = p.k / kI8Block;
    const int64_t b_row = (int64_t)group * p.n + min(col0 + lrow, p.n - 1);
    const int8_t *const b = p.B.q + b_row * p.B.ld + quarter * 16;
    const int col = col0 + quarter * 4, valid = p.n - col;

    for (int row0 = lo; row0 < hi; row0 += 16 * MT) {
        const int8_t *a[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) a[t] = p.A.q + (int64_t)min(row0 + t * 16 + lrow, hi - 1) * p.A.ld + quarter * 16;
        f8_v4i acc[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = f8_v4i{0, 0, 0, 0};
        for (int kb = wave * 4; kb < KB; kb += waves * 4) {
            if (kb + 4 <= whole) {
                f8_v4i x[8], y[8][MT];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int64_t at = (int64_t)kb * kI8Block + u * 64;
                    x[u] = *reinterpret_cast<const f8_v4i *>(b + at);
#pragma unroll
                    for (int t = 0; t < MT; ++t) y[u][t] = *reinterpret_cast<const f8_v4i *>(a[t] + at);
                }
#pragma unroll
                for (int u = 0; u < 8; ++u)
#pragma unroll
                    for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[u], y[u][t], acc[t], 0, 0, 0);
                continue;
            }
            // The blocks at the end of k, two at a time: chunks of 16 bytes that begin behind k are read as the row's last one, and A's are cut at k.
            const int last = (p.k - 1) / 16 * 16 - quarter * 16;
            for (int u0 = 0; u0 < 8 && kb * kI8Block + u0 * 64 < p.k; u0 += 4) {
                f8_v4i x[4], y[4][MT];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int64_t at = min(kb * kI8Block + (u0 + u) * 64, last);
                    x[u] = *reinterpret_cast<const f8_v4i *>(b + at);
#pragma unroll
                    for (int t = 0; t < MT; ++t) y[u][t] = *reinterpret_cast<const f8_v4i *>(a[t] + at);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int left = p.k - kb * kI8Block - (u0 + u) * 64 - quarter * 16;
#pragma unroll
                    for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[u], f8_keep(y[u][t], left), acc[t], 0, 0, 0);
                }
            }
        }
        if (row0 > lo) __syncthreads();                        // (the sums of the rows before have been read)
#pragma unroll
        for (int t = 0; t < MT; ++t) sums[(wave * MT + t) * 64 + lane] = acc[t];
        __syncthreads();
        for (int t = wave; t < MT; t += waves) {
            const int row = row0 + t * 16 + lrow;
            f8_v4i s{0, 0, 0, 0};
            for (int w = 0; w < waves; ++w) s += sums[(w * MT + t) * 64 + lane];
            if (row >= hi || valid <= 0) continue;
            const int x[4] = {s[0], s[1], s[2], s[3]};
            i8_finish_row<4>(p.out, (int64_t)row * p.out.ldc + col, x, p.A.scale[row], p.B.scale + (int64_t)group * p.n + col, valid);
        }
    }
}

template <int MT, I8Mode MODE>
hipError_t launch(const I8Args &args, hipStream_t stream) {
    const int groups = (args.k + 4 * kI8Block - 1) / (4 * kI8Block);
    const int waves = groups <= 1 ? 1 : groups <= 2 ? 2 : groups <= 4 ? 4 : kWaves;
    hipLaunchKernelGGL((k_i8_thin<MT, MODE>), dim3((unsigned)i8_tiles(MODE, I8Form::kThin, args)), dim3(waves * 64), (size_t)waves * MT * 1024, stream, args);
    return hipGetLastError();
}

template <I8Mode MODE>
hipError_t launch_rows(const I8Args &args, int rows, hipStream_t stream) {
    return rows <= 16 ? launch<1, MODE>(args, stream) : rows <= 32 ? launch<2, MODE>(args, stream) : launch<4, MODE>(args, stream);
}

}  // namespace

hipError_t launch_i8_thin(I8Mode mode, const I8Args &args, hipStream_t stream) {
    return mode == I8Mode::kDense ? launch_rows<I8Mode::kDense>(args, args.m, stream)
                                  : launch<1, I8Mode::kRows>(args, stream);
}

}  // namespace oz2
