// Products of E4M3 matrices with a power of two per block of 128, C = A B^T, by tiles of C, and the gated block on the same core.
//
// sum_h a_ih b_jh = sum over blocks of 2^(sa + sb) sum within the block: v_mfma_scale_f32_16x16x128_f8f6f4 takes one block of 128 of
// 16 rows by 16 columns with both scales as E8M0 bytes, so the sums stay in its binary32 accumulators from the first block to the last.
// The matrix core aligns the products of 8 consecutive k to the largest of them and cuts them towards zero at 2^-13 of it (measured;
// 1.4e-5 of the norm of the result for normal data, the same for the instructions with k = 32 and 64), then adds groups and accumulator in
// binary32; the E4M3 numbers themselves are rounded at 2^-4.
//
// Rows of A and B lie as the caller has them.  A stage of LDS holds the 128 bytes of a block of every row of the tile; the 16-byte
// chunk c of row r is at place c ^ (r / 2 % 8), which gives every 16 lanes that LDS serves together 16 different places (two rows
// cover all banks).  Rows beyond the matrix are read as its last one and their results dropped; in the last block, chunks
// beyond k are read as the row's last one and then cleared in LDS, in both factors, since 0 times what lies there may be NaN.
#include "oz2_epilogue.hpp"
#include "oz2_f8_device.hpp"

namespace oz2 {
namespace {

typedef __attribute__((address_space(3))) void *lds_ptr_t;

extern __shared__ f8_v4i f8_lds[];

// WM x WN wavefronts with FM x FN blocks of 16 x 16 each.  GATED: the columns of a wavefront's blocks j < FN / 2 come from the first
// weight, those of block j + FN / 2 are the same columns of the second one.
template <int WM, int WN, int FM, int FN, int STAGES, bool GATED>
struct F8Core {
    static constexpr int WAVES = WM * WN, THREADS = WAVES * 64;
    static constexpr int BM = WM * FM * 16, BN = WN * FN * 16;            // rows of A and of B in a stage
    static constexpr int ROWS = BM + BN, STAGE_BYTES = ROWS * 128;
    static constexpr int LOADS = ROWS / 8 / WAVES, A_LOADS = BM / 8 / WAVES;
    static constexpr int COLS = GATED ? BN / 2 : BN, FC = GATED ? FN / 2 : FN;   // columns of C of a tile; blocks of a wavefront
    static constexpr int GROUPS = (STAGES + 3) / 4 + 1;                   // of four blocks' scales that are in flight or in use
    static constexpr size_t LDS_BYTES = STAGES * STAGE_BYTES + GROUPS * ROWS * 4;
    static_assert(ROWS <= THREADS && ROWS % 64 == 0 && WAVES % 2 == 0 && BM % (8 * WAVES) == 0 && LOADS * (STAGES - 2) < 64, "");
};

// At most N loads of this wavefront outstanding, for one of several N; own LDS reads done; then all wavefronts meet.
template <int EACH, int MOST>
__device__ __forceinline__ void wait_ahead_and_meet(int ahead) {
    if (MOST > 0 && ahead < MOST) {                                        // uniform: the last blocks of a range
        if constexpr (MOST > 0) wait_ahead_and_meet<EACH, MOST - 1>(ahead);
        return;
    }
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(EACH * MOST) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

template <int WM, int WN, int FM, int FN, int STAGES, int PER_SIMD, bool GATED>
__global__ __launch_bounds__(WM *WN * 64, PER_SIMD) void k_f8_tiles(F8Args p, TileMap map) {
    typedef F8Core<WM, WN, FM, FN, STAGES, GATED> C;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN, lrow = lane & 15, quarter = lane >> 4;
    int range, tr, tc;
    map_tile(map, (int)blockIdx.x, range, tr, tc);
    const int row0 = tr * C::BM, col0 = tc * C::COLS;
    const int rows = min(C::BM, p.m - row0), cols = min(C::COLS, p.n - col0);
    const int KB = (p.k + kF8Block - 1) / kF8Block, kb0 = range * p.kb_each, kb1 = min(kb0 + p.kb_each, KB);

    // Row of B for row r of that part of a stage: the column of C and, gated, which of the two weights.
    const auto b_column = [](int r) { return GATED ? r / (FN * 16) * (FN * 8) + r % (FN * 8) : r; };
    const auto b_second = [](int r) { return GATED && r / (FN * 8) % 2; };

    // Load H of this wavefront takes the 8 rows from 8 (H WAVES + wave) on; a lane 16 bytes of one.
    const uint8_t *const a_base = p.A.q + (int64_t)row0 * p.A.ld, *const b_base = p.B.q + (int64_t)col0 * p.B.ld;
    const uint8_t *const b_base2 = GATED ? b_base + (int64_t)p.up * p.B.ld : b_base;
    const int chunk = (lane & 7) ^ ((wave & 1) * 4 + quarter);
    uint32_t offset[C::LOADS];
#pragma unroll
    for (int h = 0; h < C::LOADS; ++h) {
        const int r = (h * C::WAVES + wave) * 8 + (lane >> 3);
        offset[h] = h < C::A_LOADS ? (uint32_t)min(r, rows - 1) * (uint32_t)p.A.ld : (uint32_t)min(b_column(r - C::BM), cols - 1) * (uint32_t)p.B.ld;
        offset[h] += chunk * 16;
    }
    const int in_last = p.k - (KB - 1) * kF8Block;                         // of the last block, 1 to 128
    const int to_last_chunk = (min(chunk, (in_last - 1) / 16) - chunk) * 16;
    // A lane's scales: four blocks of one row, those of all rows are fetched by the workgroup together.
    const uint8_t *scales;
    {
        const int r = min((int)threadIdx.x, C::ROWS - 1);
        if (r < C::BM) scales = p.A.scale + (int64_t)((row0 + min(r, rows - 1)) >> p.A.shift) * p.A.ld_scale;
        else {
            const int br = col0 + min(b_column(r - C::BM), cols - 1) + (b_second(r - C::BM) ? p.up : 0);
            scales = p.B.scale + (int64_t)(br >> p.B.shift) * p.B.ld_scale;
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)f8_lds;
    int want = kb0, want_stage = 0, want_group = 0;                        // the block that is requested next, and where it goes
    const auto request = [&]() {
        if (want >= kb1) return;                                           // uniform
        const uint32_t back = want == KB - 1 ? (uint32_t)to_last_chunk : 0u;
        if ((want & 3) == 0) {
            if (wave * 64 < C::ROWS) {                                     // uniform
                const uint32_t to = lds0 + STAGES * C::STAGE_BYTES + (want_group * C::ROWS + wave * 64) * 4;
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(scales + want) : "memory");
            }
            want_group = want_group + 1 == C::GROUPS ? 0 : want_group + 1;
        }
#pragma unroll
        for (int h = 0; h < C::LOADS; ++h) {
            const bool second = h >= C::A_LOADS && b_second((h * C::WAVES + wave) * 8 - C::BM);       // uniform
            const uint8_t *const base = (h < C::A_LOADS ? a_base : second ? b_base2 : b_base) + (int64_t)want * kF8Block;
            const uint32_t to = lds0 + want_stage * C::STAGE_BYTES + (h * C::WAVES + wave) * 1024;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset[h] + back), "s"(base) : "memory");
        }
        ++want;
        want_stage = want_stage + 1 == STAGES ? 0 : want_stage + 1;
    };

    f8_v4f acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f8_v4f{0.f, 0.f, 0.f, 0.f};
    const char *const lds = reinterpret_cast<const char *>(f8_lds);
    const int swizzled = (quarter ^ (lane >> 1 & 7)) * 16;
    const int a_addr = (wm * FM * 16 + lrow) * 128 + swizzled, b_addr = (C::BM + wn * FN * 16 + lrow) * 128 + swizzled;
    struct Fragments {
        f8_v8i a[FM], b[FN];
        int sa[FM], sb[FN];
    };
    int stage = 0, group = 0;                                              // of the block that is read next
    const auto read = [&](Fragments &f, const Fragments &before, int kb) {
        const auto fragment = [&](int addr, int i) {
            const char *const at = lds + stage * C::STAGE_BYTES + i * 2048;
            return f8_join(*reinterpret_cast<const f8_v4i *>(at + addr), *reinterpret_cast<const f8_v4i *>(at + (addr ^ 64)));
        };
#pragma unroll
        for (int i = 0; i < FM; ++i) f.a[i] = fragment(a_addr, i);
#pragma unroll
        for (int j = 0; j < FN; ++j) f.b[j] = fragment(b_addr, j);
        if ((kb & 3) == 0) {
            const int *const s = reinterpret_cast<const int *>(lds + STAGES * C::STAGE_BYTES) + group * C::ROWS;
#pragma unroll
            for (int i = 0; i < FM; ++i) f.sa[i] = s[(wm * FM + i) * 16 + lrow];
#pragma unroll
            for (int j = 0; j < FN; ++j) f.sb[j] = s[C::BM + (wn * FN + j) * 16 + lrow];
            group = group + 1 == C::GROUPS ? 0 : group + 1;
        } else {
#pragma unroll
            for (int i = 0; i < FM; ++i) f.sa[i] = (int)((uint32_t)before.sa[i] >> 8);
#pragma unroll
            for (int j = 0; j < FN; ++j) f.sb[j] = (int)((uint32_t)before.sb[j] >> 8);
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    };
    // Waits until block kb is there; whoever comes here has read all blocks before it.
    const auto arrive = [&](int kb) {
        wait_ahead_and_meet<C::LOADS, STAGES - 2>(want - 1 - kb);
        if (kb == KB - 1 && in_last < kF8Block) {                          // what lies behind k, of this thread's row
            if ((int)threadIdx.x < C::ROWS) {
                const int r = (int)threadIdx.x, from = in_last >> 4, f = r >> 1 & 7;
                f8_v4i *const row = f8_lds + stage * (C::STAGE_BYTES / 16) + r * 8;
                row[from ^ f] = f8_keep(row[from ^ f], in_last & 15);
                for (int c = from + 1; c < 8; ++c) row[c ^ f] = f8_v4i{0, 0, 0, 0};
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
    };
    const auto multiply = [&](const Fragments &f) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[i][j] = f8_mfma(f.b[j], f.a[i], acc[i][j], f.sb[j], f.sa[i]);
    };
    // The fragments of a block are read during the MFMAs of the one before; STAGES - 1 blocks are in flight.
    if (kb0 < kb1) {
        Fragments f, g;
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) request();
        arrive(kb0);
        request();
        read(f, f, kb0);
        for (int kb = kb0 + 1;; kb += 2) {
            if (kb < kb1) {
                arrive(kb);
                request();
                read(g, f, kb);
            }
            multiply(f);
            if (kb >= kb1) break;
            if (kb + 1 < kb1) {
                arrive(kb + 1);
                request();
                read(f, g, kb + 1);
            }
            multiply(g);
            if (kb + 1 >= kb1) break;
        }
    }

    const F8Out &o = p.out;
    // N numbers of a row, at a column that is a multiple of N.
    const auto emit = [&](auto &x, auto &u, int row, int col) {
        constexpr int N = sizeof(x) / sizeof(x[0]);
        const int valid = row < p.m ? p.n - col : 0;
        if (valid <= 0) return;
        if (o.planes) {
            const int64_t at = range * o.plane + (int64_t)row * o.ldp + col;
            f8_store_row<N>(o.planes, kF8F32, at, x, valid);
            if (GATED) f8_store_row<N>(o.planes, kF8F32, at + o.ldp / 2, u, valid);
        } else if constexpr (!GATED) f8_update_row<N>(o, (int64_t)row * o.ldc + col, x, valid);
        else {
            if (o.Z) {
                f8_store_row<N>(o.Z, o.type, (int64_t)row * o.ldz + col, x, valid);
                f8_store_row<N>(o.Z, o.type, (int64_t)row * o.ldz + p.up + col, u, valid);
            }
            f8_gated(x, u, o.act);
            f8_store_row<N>(o.C, o.type, (int64_t)row * o.ldc + col, x, valid);
        }
    };
    if constexpr (C::FC == 1) {                                            // 4 numbers of a row per lane, as they are
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            float x[4], u[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = acc[i][0][r];
                u[r] = GATED ? acc[i][FN - 1][r] : 0.f;
            }
            emit(x, u, row0 + (wm * FM + i) * 16 + lrow, col0 + wn * 16 + quarter * 4);
        }
    } else {
        // Four blocks at a time, exchanged so that quarter q of the wavefront has 16 columns of block q's rows: blocks (i, j) to (i, j + 3),
        // or, of two columns of blocks, (i, 0), (i, 1), (i + 1, 0), (i + 1, 1).
        constexpr int GI = C::FC >= 4 ? 1 : 2, GJ = 4 / GI;
        static_assert(FM % GI == 0 && C::FC % GJ == 0, "");
        const auto gathered = [&](int i, int j, float(&x)[16]) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float f[4] = {acc[i][j][r], acc[i][j + 1][r], acc[i + (GI - 1)][GJ == 4 ? j + 2 : j][r], acc[i + (GI - 1)][GJ == 4 ? j + 3 : j + 1][r]};
                uint32_t d[4];                                             // (a bit cast of an element of a vector takes the first one)
#pragma unroll
                for (int q = 0; q < 4; ++q) d[q] = __builtin_bit_cast(uint32_t, f[q]);
                const exchanged_t e = exchange_quarters(d);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int w = e[q];
                    x[4 * q + r] = __builtin_bit_cast(float, w);
                }
            }
        };
#pragma unroll
        for (int i = 0; i < FM; i += GI)
#pragma unroll
            for (int j = 0; j < C::FC; j += GJ) {
                float x[16], u[16];
                gathered(i, j, x);
                if constexpr (GATED) gathered(i, j + C::FC, u);
                emit(x, u, row0 + (wm * FM + i + quarter / GJ) * 16 + lrow, col0 + (wn * C::FC + j + quarter % GJ) * 16);
            }
    }
}

// The sums of the K ranges, in ascending order, and what the tiles do with a sum.  A thread has 4 columns of a row.
template <bool GATED>
__global__ __launch_bounds__(256) void k_f8_ranges(F8Args p) {
    const int per_row = (p.n + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / per_row;
    if (row >= p.m) return;
    const int col = (int)(id - row * per_row) * 4, valid = p.n - col;
    const F8Out &o = p.out;
    const float *const from = o.planes + row * o.ldp + col;
    f8_v4f s{0.f, 0.f, 0.f, 0.f}, t{0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < p.ranges; r0 += 4) {                 // four loads at a time: one after the other costs a way to memory each
        f8_v4f x[4], y[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float *const plane = from + (int64_t)min(r0 + r, p.ranges - 1) * o.plane;
            x[r] = *reinterpret_cast<const f8_v4f *>(plane);
            if (GATED) y[r] = *reinterpret_cast<const f8_v4f *>(plane + o.ldp / 2);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r0 + r < p.ranges) {
                s += x[r];
                if (GATED) t += y[r];
            }
    }
    float x[4] = {s[0], s[1], s[2], s[3]};
    if constexpr (!GATED) f8_update_row<4>(o, row * o.ldc + col, x, valid);
    else {
        float u[4] = {t[0], t[1], t[2], t[3]};
        if (o.Z) {
            f8_store_row<4>(o.Z, o.type, row * o.ldz + col, x, valid);
            f8_store_row<4>(o.Z, o.type, row * o.ldz + p.up + col, u, valid);
        }
        f8_gated(x, u, o.act);
        f8_store_row<4>(o.C, o.type, row * o.ldc + col, x, valid);
    }
}

template <int WM, int WN, int FM, int FN, int STAGES, int PER_SIMD, bool GATED>
hipError_t launch_tiles(const F8Args &args, hipStream_t stream) {
    typedef F8Core<WM, WN, FM, FN, STAGES, GATED> C;
    static thread_local int attr_device = -1;                // the attribute is per device (set again per thread: harmless)
    int dev = -1;
    if (hipError_t e = hipGetDevice(&dev)) return e;
    if (attr_device != dev) {
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_f8_tiles<WM, WN, FM, FN, STAGES, PER_SIMD, GATED>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::LDS_BYTES)) return e;
        attr_device = dev;
    }
    const int tiles_m = (args.m + C::BM - 1) / C::BM, tiles_n = (args.n + C::COLS - 1) / C::COLS;
    const TileMap map = make_tile_map(tiles_m, tiles_n, tiles_m * tiles_n * args.ranges);
    hipLaunchKernelGGL((k_f8_tiles<WM, WN, FM, FN, STAGES, PER_SIMD, GATED>), dim3((unsigned)map.total), dim3(C::THREADS), C::LDS_BYTES, stream, args, map);
    return hipGetLastError();
}

// Tiles of 64 x 64 by four wavefronts of 32 x 32, with four stages (two workgroups share a unit's LDS) while all tiles fit the device at
// once and the way of a block to LDS counts, else with two (four workgroups).  Four | two, us: 512 x 512 x 4096 13.6 | 18.8, 1400 x 1400 x 4096 (484
// tiles) 18.8 | 21.1, 1500 x 1500 x 4096 (576) 28.0 | 22.1, 2000 x 1800 x 300 9.6 | 7.9.  Tiles of 64 x 128 with two stages.
// 500 x 300 x 777 6.2 us, 1024^3 5.7 us, 2048^3 15.6 us (1.1 PFLOP/s): bound by the ways to memory and LDS one after the other, launch included.
template <bool GATED>
hipError_t launch_form(const F8Args &args, const F8Plan &plan, hipStream_t stream) {
    const bool deep = f8_items(plan.form, args.m, args.n, GATED) * args.ranges <= 512;
    if (hipError_t e = plan.form == F8Form::kLarge    ? launch_f8_wide(args, GATED, stream)
                       : plan.form == F8Form::kMiddle ? launch_tiles<2, 2, 2, 4, 2, 2, GATED>(args, stream)
                       : deep                         ? launch_tiles<2, 2, 2, 2, 4, 2, GATED>(args, stream)
                                                      : launch_tiles<2, 2, 2, 2, 2, 4, GATED>(args, stream)) return e;
    if (args.ranges == 1) return hipSuccess;
    const int64_t threads = (int64_t)args.m * ((args.n + 3) / 4);
    hipLaunchKernelGGL(k_f8_ranges<GATED>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, args);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_product(const F8Args &args, const F8Plan &plan, bool gated, hipStream_t stream) {
    if (plan.form == F8Form::kThin) return launch_f8_thin(args, gated, stream);
    return gated ? launch_form<true>(args, plan, stream) : launch_form<false>(args, plan, stream);
}

}  // namespace oz2
