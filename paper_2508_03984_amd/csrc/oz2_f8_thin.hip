// Products of E4M3 matrices with few rows of A (tokens that are decoded): every element of B is read once, straight into the registers of
// the matrix instruction, and C has no other work.  A workgroup takes 16 columns of C (gated: of both weights), its wavefronts
// take groups of 4 blocks of k in turn and add their sums through LDS in ascending order.
//
// 1 x 8192 x 8192 13.7 us, 4.9 TB/s; 1 x 16384 x 16384 56 us, 4.8 TB/s; gated, 4 x 16384 x 4096 29.2 us, 4.6 TB/s.  Bound: HBM (the bytes of B);
// with more rows what a compute unit reads through its caches, 16 bytes a lane from rows of their own (23 x 84 x 11286 15 us).
#include "oz2_f8_device.hpp"

namespace oz2 {
namespace {

constexpr int kWaves = 8;                                     // of a workgroup at most (with 16, 1 x 16 x 16384 takes as long: its unit's loads bound it)

// MT blocks of 16 rows of A.
template <int MT, bool GATED>
__global__ __launch_bounds__(kWaves * 64) void k_f8_thin(F8Args p) {
    constexpr int SIDES = GATED ? 2 : 1;
    extern __shared__ f8_v4f sums[];                          // [wavefronts][SIDES * MT][64]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = (int)blockDim.x >> 6;
    const int lrow = lane & 15, quarter = lane >> 4;
    const int col0 = (int)blockIdx.x * 16;
    const int KB = (p.k + kF8Block - 1) / kF8Block, whole = p.k / kF8Block;

    const uint8_t *b[SIDES], *b_scale[SIDES], *a[MT], *a_scale[MT];
#pragma unroll
    for (int s = 0; s < SIDES; ++s) {
        const int row = min(col0 + lrow, p.n - 1) + (s ? p.up : 0);
        b[s] = p.B.q + (int64_t)row * p.B.ld + quarter * 16;
        b_scale[s] = p.B.scale + (int64_t)(row >> p.B.shift) * p.B.ld_scale;
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int row = min(t * 16 + lrow, p.m - 1);
        a[t] = p.A.q + (int64_t)row * p.A.ld + quarter * 16;
        a_scale[t] = p.A.scale + (int64_t)(row >> p.A.shift) * p.A.ld_scale;
    }
    f8_v4f acc[SIDES][MT];
#pragma unroll
    for (int s = 0; s < SIDES; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[s][t] = f8_v4f{0.f, 0.f, 0.f, 0.f};

    for (int kb = wave * 4; kb < KB; kb += waves * 4) {
        int sb[SIDES], sa[MT];
#pragma unroll
        for (int s = 0; s < SIDES; ++s) sb[s] = *reinterpret_cast<const int *>(b_scale[s] + kb);
#pragma unroll
        for (int t = 0; t < MT; ++t) sa[t] = *reinterpret_cast<const int *>(a_scale[t] + kb);
        const auto multiply = [&](const f8_v8i(&x)[SIDES], const f8_v8i(&y)[MT], int u) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int s = 0; s < SIDES; ++s) acc[s][t] = f8_mfma(x[s], y[t], acc[s][t], (int)((uint32_t)sb[s] >> 8 * u), (int)((uint32_t)sa[t] >> 8 * u));
        };
        if (kb + 4 <= whole) {
            f8_v8i x[4][SIDES], y[4][MT];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t at = (int64_t)(kb + u) * kF8Block;
#pragma unroll
                for (int s = 0; s < SIDES; ++s)
                    x[u][s] = f8_join(*reinterpret_cast<const f8_v4i *>(b[s] + at), *reinterpret_cast<const f8_v4i *>(b[s] + at + 64));
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    y[u][t] = f8_join(*reinterpret_cast<const f8_v4i *>(a[t] + at), *reinterpret_cast<const f8_v4i *>(a[t] + at + 64));
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) multiply(x[u], y[u], u);
            continue;
        }
        // The blocks at the end of k, two at a time: chunks of 16 bytes that begin behind k are read as the row's last one, and all are cut at k.
        const int last = (p.k - 1) / 16 * 16 - quarter * 16;
        for (int u0 = 0; u0 < 4 && kb + u0 < KB; u0 += 2) {
            f8_v4i x[2][SIDES][2], y[2][MT][2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int64_t at = min((kb + u0 + u) * kF8Block + half * 64, last);
#pragma unroll
                    for (int s = 0; s < SIDES; ++s) x[u][s][half] = *reinterpret_cast<const f8_v4i *>(b[s] + at);
#pragma unroll
                    for (int t = 0; t < MT; ++t) y[u][t][half] = *reinterpret_cast<const f8_v4i *>(a[t] + at);
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (kb + u0 + u >= KB) break;                 // uniform (the scales behind k may be anything, NaN too)
                const int left = p.k - (kb + u0 + u) * kF8Block - quarter * 16;
                f8_v8i xs[SIDES], ys[MT];
#pragma unroll
                for (int s = 0; s < SIDES; ++s) xs[s] = f8_join(f8_keep(x[u][s][0], left), f8_keep(x[u][s][1], left - 64));
#pragma unroll
                for (int t = 0; t < MT; ++t) ys[t] = f8_join(f8_keep(y[u][t][0], left), f8_keep(y[u][t][1], left - 64));
                multiply(xs, ys, u0 + u);
            }
        }
    }

#pragma unroll
    for (int s = 0; s < SIDES; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t) sums[(wave * SIDES * MT + s * MT + t) * 64 + lane] = acc[s][t];
    __syncthreads();
    const F8Out &o = p.out;
    const int col = col0 + quarter * 4, valid = p.n - col;
    for (int t = wave; t < MT; t += waves) {
        const int row = t * 16 + lrow;
        f8_v4f s{0.f, 0.f, 0.f, 0.f}, v{0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < waves; ++w) {
            s += sums[(w * SIDES * MT + t) * 64 + lane];
            if (GATED) v += sums[(w * SIDES * MT + MT + t) * 64 + lane];
        }
        if (row >= p.m || valid <= 0) continue;
        float x[4] = {s[0], s[1], s[2], s[3]};
        if constexpr (!GATED) f8_update_row<4>(o, row * o.ldc + col, x, valid);
        else {
            float u[4] = {v[0], v[1], v[2], v[3]};
            if (o.Z) {
                f8_store_row<4>(o.Z, o.type, row * o.ldz + col, x, valid);
                f8_store_row<4>(o.Z, o.type, row * o.ldz + p.up + col, u, valid);
            }
            f8_gated(x, u, o.act);
            f8_store_row<4>(o.C, o.type, row * o.ldc + col, x, valid);
        }
    }
}

template <int MT, bool GATED>
hipError_t launch(const F8Args &args, hipStream_t stream) {
    const int groups = (args.k + 4 * kF8Block - 1) / (4 * kF8Block);
    const int waves = groups <= 1 ? 1 : groups <= 2 ? 2 : groups <= 4 ? 4 : kWaves;
    const size_t lds_bytes = (size_t)waves * MT * (GATED ? 2 : 1) * 1024;
    hipLaunchKernelGGL((k_f8_thin<MT, GATED>), dim3((unsigned)((args.n + 15) / 16)), dim3(waves * 64), lds_bytes, stream, args);
    return hipGetLastError();
}

template <bool GATED>
hipError_t launch_rows(const F8Args &args, hipStream_t stream) {
    return args.m <= 16 ? launch<1, GATED>(args, stream) : args.m <= 32 ? launch<2, GATED>(args, stream) : launch<4, GATED>(args, stream);
}

}  // namespace

hipError_t launch_f8_thin(const F8Args &args, bool gated, hipStream_t stream) {
    return gated ? launch_rows<true>(args, stream) : launch_rows<false>(args, stream);
}

}  // namespace oz2
