// Products of matrices in 8-bit integers with a scale for each row, C_ij = alpha a_i b_j sum_h A_ih B_jh + beta C_ij, by tiles of C: alone (kDense), the rows of A by
// group, each with its own B (kRows), or the columns of both by group, each with its own C (kSums).
//
// v_mfma_i32_16x16x64_i8 adds 64 products per entry of a 16 x 16 block to its int32 accumulators, exactly; the two scales are applied once, to the sum.
//
// Rows of A and B lie as the caller has them.  A stage of LDS holds 128 bytes of every row of the tile; the 16-byte chunk c of row r is at place
// c ^ (r / 2 % 8), which gives every 16 lanes that LDS serves together 16 different places (two rows cover all banks).  Rows beyond the matrix or
// the group are read as its last one and their results dropped; in the last block of k, chunks beyond k are read as the row's last one and
// then cleared in LDS, in A only, since 0 times whatever B has there is 0.
//
// The scales of a tile's rows and columns are fetched before its sums and lie in LDS behind the stages: from memory, in the store phase, they cost 64 x 64 tiles their registers
// (2048^3 26 -> 16 us).  500 x 300 x 777 5.7 us a call, 1024 x 4096 x 4096 23.5 us (1.5 POP/s), 24 experts of 1500 x 1111 and 1332 rows 11.4 us (4.0 TB/s): bound by the ways to memory and LDS one after
// the other, and by HBM where an expert has few rows.
#include "oz2_epilogue.hpp"
#include "oz2_i8_device.hpp"

namespace oz2 {
namespace {

typedef __attribute__((address_space(3))) void *lds_ptr_t;

extern __shared__ f8_v4i i8_lds[];

// WM x WN wavefronts with FM x FN blocks of 16 x 16 each.
template <int WM, int WN, int FM, int FN, int STAGES>
struct I8Core {
    static constexpr int WAVES = WM * WN, THREADS = WAVES * 64;
    static constexpr int BM = WM * FM * 16, BN = WN * FN * 16;
    static constexpr int ROWS = BM + BN, STAGE_BYTES = ROWS * 128;
    static constexpr int LOADS = ROWS / 8 / WAVES, A_LOADS = BM / 8 / WAVES;
    static constexpr size_t LDS_BYTES = STAGES * STAGE_BYTES + ROWS * 4;  // the scales of the rows behind the stages
    static_assert(ROWS <= THREADS && WAVES % 2 == 0 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && LOADS * (STAGES - 2) < 64, "");
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

// What a workgroup computes: rows x cols entries (at most a tile) over the blocks kb0 to kb1 - 1 of k, of which the last one of the row ends after k.
struct Tile {
    const int8_t *a, *b;                                                   // the first rows of both
    const float *scale_a, *scale_b;
    int rows, cols, k, kb0, kb1;
    int64_t c_row;                                                         // row of C, column
    int c_col, range;
    bool lost;                                                             // more columns than int32 sums can hold for certain: NaN
};

// The places of a group's tiles: bands of 8 rows of tiles, within a band column by column, so that the 32 workgroups which an XCD runs at a time share A's and B's rows.
__device__ __forceinline__ void place_in_group(uint32_t piece, uint32_t units, uint32_t tiles_n, int &tr, int &tc) {
    const uint32_t band = piece / (8 * tiles_n), left = piece - band * 8 * tiles_n, high = min(8u, units - band * 8);
    tc = (int)(left / high);
    tr = (int)(band * 8 + left - (uint32_t)tc * high);
}

// LAST: of the large tiles that the launch before has left, BM x BN parts; the map is that of the large tiles.
template <I8Mode MODE, int BM, int BN, bool LAST>
__device__ __forceinline__ bool find_tile(const I8Args &p, const TileMap &map, int id, Tile &t) {
    constexpr int HIGH = LAST ? 256 : BM, BROAD = LAST ? 256 : BN, PARTS = HIGH * BROAD / (BM * BN), ACROSS = BROAD / BN;
    t.lost = false;
    t.range = 0;
    if constexpr (MODE == I8Mode::kRows) {
        const uint32_t tiles_n = (uint32_t)(p.n + BROAD - 1) / BROAD;
        I8Place at;
        if (!LAST && p.ranges > 1) {                                       // (the grid has a part of its own for each, of whole eights)
            const int part = (int)gridDim.x / p.ranges;
            t.range = id / part;
            id -= t.range * part;
        }
        if constexpr (LAST) {
            const bool found = i8_find_place(p.groups, HIGH, tiles_n, [&](uint32_t total) {
                const uint32_t share = (total + 7) / 8, left = i8_left_over(share, (uint32_t)p.turn / 8), local = (uint32_t)(id >> 3) / PARTS;
                return local < left ? (uint32_t)(id & 7) * share + share - left + local : ~0u;
            }, at);
            if (!found) return false;
        } else if (!i8_find(p.groups, HIGH, tiles_n, (uint32_t)id, at)) return false;
        int tr, tc;
        place_in_group(at.piece, at.units, tiles_n, tr, tc);
        const int part = LAST ? (id >> 3) % PARTS : 0, row0 = at.span.lo + tr * HIGH + part / ACROSS * BM, col0 = tc * BROAD + part % ACROSS * BN;
        if (LAST && (row0 >= at.span.hi || col0 >= p.n)) return false;
        const int64_t b_row = (int64_t)at.span.group * p.n + col0;
        t.rows = min(BM, at.span.hi - row0);
        t.cols = min(BN, p.n - col0);
        t.a = p.A.q + row0 * p.A.ld;
        t.b = p.B.q + b_row * p.B.ld;
        t.scale_a = p.A.scale + row0;
        t.scale_b = p.B.scale + b_row;
        t.k = p.k;
        t.kb0 = t.range * p.kb_each;
        t.kb1 = min(t.kb0 + p.kb_each, (p.k + kI8Block - 1) / kI8Block);
        t.c_row = row0;
        t.c_col = col0;
    } else {
        int s, tr, tc;
        const int first_left = LAST ? map.total - (int)i8_left_over((uint32_t)map.total, (uint32_t)p.turn) : 0, part = LAST ? id % PARTS : 0;
        map_tile(map, LAST ? first_left + id / PARTS : id, s, tr, tc);
        const int row0 = tr * HIGH + part / ACROSS * BM, col0 = tc * BROAD + part % ACROSS * BN;
        if (LAST && (row0 >= p.m || col0 >= p.n)) return false;
        t.rows = min(BM, p.m - row0);
        t.cols = min(BN, p.n - col0);
        t.c_col = col0;
        int64_t first = 0, scales_a = 0, scales_b = 0;
        if constexpr (MODE == I8Mode::kDense) {
            t.k = p.k;
            const int KB = (p.k + kI8Block - 1) / kI8Block;
            t.kb0 = s * p.kb_each;
            t.kb1 = min(t.kb0 + p.kb_each, KB);
            t.range = s;
            t.c_row = row0;
        } else {
            if (p.ranges > 1) {
                t.range = s / p.groups.groups;
                s -= t.range * p.groups.groups;
            }
            const I8Span span = i8_span(p.groups, s);
            if (p.only_short && i8_by_large_tiles(span.hi - span.lo)) return false;
            first = i8_first_col(span);
            scales_a = s * p.A.ld_scale;
            scales_b = s * p.B.ld_scale;
            t.lost = span.hi - span.lo > kI8MaxK;
            const int KB = t.lost ? 0 : (span.hi - span.lo + kI8Block - 1) / kI8Block, each = p.ranges > 1 ? (KB + p.ranges - 1) / p.ranges : KB;
            t.kb0 = min(t.range * each, KB);
            t.kb1 = min(t.kb0 + each, KB);
            t.k = KB * kI8Block;                                           // (zeros follow up to there)
            t.c_row = (int64_t)s * p.m + row0;
        }
        t.a = p.A.q + row0 * p.A.ld + first;
        t.b = p.B.q + col0 * p.B.ld + first;
        t.scale_a = p.A.scale + scales_a + row0;
        t.scale_b = p.B.scale + scales_b + col0;
    }
    return true;
}

template <int WM, int WN, int FM, int FN, int STAGES, int PER_SIMD, I8Mode MODE, bool LAST>
__global__ __launch_bounds__(WM *WN * 64, PER_SIMD) void k_i8_tiles(I8Args p, TileMap map) {
    typedef I8Core<WM, WN, FM, FN, STAGES> C;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN, lrow = lane & 15, quarter = lane >> 4;
    Tile t;
    if (!find_tile<MODE, C::BM, C::BN, LAST>(p, map, (int)blockIdx.x, t)) return;
    const int KB = (t.k + kI8Block - 1) / kI8Block, kb0 = t.kb0, kb1 = t.kb1;

    const bool none = kb0 >= kb1;
    float scale = 0.0f;                                                    // of a row of A or B for each thread, which all need after the sums
    if (!none && (int)threadIdx.x < C::ROWS)
        scale = (int)threadIdx.x < C::BM ? t.scale_a[min((int)threadIdx.x, t.rows - 1)] : t.scale_b[min((int)threadIdx.x - C::BM, t.cols - 1)];

    // Load H of this wavefront takes the 8 rows from 8 (H WAVES + wave) on; a lane 16 bytes of one.
    const int chunk = (lane & 7) ^ ((wave & 1) * 4 + quarter);
    uint32_t offset[C::LOADS];
#pragma unroll
    for (int h = 0; h < C::LOADS; ++h) {
        const int r = (h * C::WAVES + wave) * 8 + (lane >> 3);
        offset[h] = h < C::A_LOADS ? (uint32_t)min(r, t.rows - 1) * (uint32_t)p.A.ld : (uint32_t)min(r - C::BM, t.cols - 1) * (uint32_t)p.B.ld;
        offset[h] += chunk * 16;
    }
    const int in_last = t.k - (KB - 1) * kI8Block;                         // of the last block, 1 to 128
    const int to_last_chunk = (min(chunk, (in_last - 1) / 16) - chunk) * 16;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)i8_lds;
    int want = kb0, want_stage = 0;                                        // the block that is requested next, and where it goes
    const auto request = [&]() {
        if (want >= kb1) return;                                           // uniform
        const uint32_t back = want == KB - 1 ? (uint32_t)to_last_chunk : 0u;
#pragma unroll
        for (int h = 0; h < C::LOADS; ++h) {
            const int8_t *const base = (h < C::A_LOADS ? t.a : t.b) + (int64_t)want * kI8Block;
            const uint32_t to = lds0 + want_stage * C::STAGE_BYTES + (h * C::WAVES + wave) * 1024;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset[h] + back), "s"(base) : "memory");
        }
        ++want;
        want_stage = want_stage + 1 == STAGES ? 0 : want_stage + 1;
    };

    f8_v4i acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f8_v4i{0, 0, 0, 0};
    const char *const lds = reinterpret_cast<const char *>(i8_lds);
    const int swizzled = (quarter ^ (lane >> 1 & 7)) * 16;
    const int a_addr = (wm * FM * 16 + lrow) * 128 + swizzled, b_addr = (C::BM + wn * FN * 16 + lrow) * 128 + swizzled;
    struct Fragments {
        f8_v4i a[FM][2], b[FN][2];                                         // halves of a block of 128
    };
    int stage = 0;                                                         // of the block that is read next
    const auto read = [&](Fragments &f) {
        const char *const at = lds + stage * C::STAGE_BYTES;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int i = 0; i < FM; ++i) f.a[i][half] = *reinterpret_cast<const f8_v4i *>(at + i * 2048 + (a_addr ^ half * 64));
#pragma unroll
            for (int j = 0; j < FN; ++j) f.b[j][half] = *reinterpret_cast<const f8_v4i *>(at + j * 2048 + (b_addr ^ half * 64));
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    };
    // Waits until block kb is there; whoever comes here has read all blocks before it.
    const auto arrive = [&](int kb) {
        wait_ahead_and_meet<C::LOADS, STAGES - 2>(want - 1 - kb);
        if (kb == KB - 1 && in_last < kI8Block) {                          // what lies behind k, of this thread's row of A
            if ((int)threadIdx.x < C::BM) {
                const int r = (int)threadIdx.x, from = in_last >> 4, f = r >> 1 & 7;
                f8_v4i *const row = i8_lds + stage * (C::STAGE_BYTES / 16) + r * 8;
                row[from ^ f] = f8_keep(row[from ^ f], in_last & 15);
                for (int c = from + 1; c < 8; ++c) row[c ^ f] = f8_v4i{0, 0, 0, 0};
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
    };
    const auto multiply = [&](const Fragments &f) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int i = 0; i < FM; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.b[j][half], f.a[i][half], acc[i][j], 0, 0, 0);
    };
    // The fragments of a block are read during the MFMAs of the one before; STAGES - 1 blocks are in flight.
    if (kb0 < kb1) {
        Fragments f, g;
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) request();
        arrive(kb0);
        request();
        read(f);
        for (int kb = kb0 + 1;; kb += 2) {
            if (kb < kb1) {
                arrive(kb);
                request();
                read(g);
            }
            multiply(f);
            if (kb >= kb1) break;
            if (kb + 1 < kb1) {
                arrive(kb + 1);
                request();
                read(f);
            }
            multiply(g);
            if (kb + 1 >= kb1) break;
        }
    }

    float *const scales = reinterpret_cast<float *>(i8_lds) + STAGES * C::STAGE_BYTES / 4;
    if ((int)threadIdx.x < C::ROWS) scales[threadIdx.x] = scale;
    __syncthreads();
    F8Out o = p.out;
    if (none) o.alpha = 0.0f;                                              // no infinity or NaN from it
    // 16 numbers of a row, at a column that is a multiple of 16.
    const auto emit = [&](const int (&sum)[16], int row, int col) {
        constexpr int N = 16;
        const int valid = row < t.rows ? t.cols - col : 0;
        if (valid <= 0) return;
        if (o.planes) {                                                    // (a plane's rows are stored to a multiple of 16)
            int32_t *const to = reinterpret_cast<int32_t *>(o.planes) + t.range * o.plane + (t.c_row + row) * o.ldp + t.c_col + col;
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const f8_v4i w{sum[i], sum[i + 1], sum[i + 2], sum[i + 3]};
                *reinterpret_cast<f8_v4i *>(to + i) = w;
            }
            return;
        }
        float x[N];
        const float a = t.lost ? __builtin_nanf("") : scales[row];
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const f8_v4f b = *reinterpret_cast<const f8_v4f *>(scales + C::BM + col + i);
#pragma unroll
            for (int u = 0; u < 4; ++u) x[i + u] = (float)sum[i + u] * a * b[u];
        }
        f8_update_row<N>(o, (t.c_row + row) * o.ldc + t.c_col + col, x, valid);
    };
    // Four blocks at a time, exchanged so that quarter q of the wavefront has 16 columns of block q's rows: blocks (i, j) to (i, j + 3),
    // or, of two columns of blocks, (i, 0), (i, 1), (i + 1, 0), (i + 1, 1).
    constexpr int GI = FN >= 4 ? 1 : 2, GJ = 4 / GI;
    static_assert(FM % GI == 0 && FN % GJ == 0, "");
#pragma unroll
    for (int i = 0; i < FM; i += GI)
#pragma unroll
        for (int j = 0; j < FN; j += GJ) {
            int x[16];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t d[4] = {(uint32_t)acc[i][j][r], (uint32_t)acc[i][j + 1][r], (uint32_t)acc[i + (GI - 1)][GJ == 4 ? j + 2 : j][r],
                                       (uint32_t)acc[i + (GI - 1)][GJ == 4 ? j + 3 : j + 1][r]};
                const exchanged_t e = exchange_quarters(d);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[4 * q + r] = e[q];
            }
            emit(x, (wm * FM + i + quarter / GJ) * 16 + lrow, (wn * FN + j + quarter % GJ) * 16);
        }
}

template <int WM, int WN, int FM, int FN, int STAGES, int PER_SIMD, I8Mode MODE, bool LAST = false>
hipError_t launch_tiles(const I8Args &args, I8Form form, hipStream_t stream) {
    typedef I8Core<WM, WN, FM, FN, STAGES> C;
    static thread_local int attr_device = -1;                // the attribute is per device (set again per thread: harmless)
    int dev = -1;
    if (hipError_t e = hipGetDevice(&dev)) return e;
    if (attr_device != dev) {
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_i8_tiles<WM, WN, FM, FN, STAGES, PER_SIMD, MODE, LAST>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::LDS_BYTES)) return e;
        attr_device = dev;
    }
    constexpr int HIGH = LAST ? 256 : C::BM, BROAD = LAST ? 256 : C::BN;
    const int64_t all = i8_tiles(MODE, LAST ? I8Form::kLarge : form, args);
    // (kRows: as many as a last round that is left may have)
    const int64_t tiles = !LAST ? all : (MODE == I8Mode::kDense ? (int64_t)i8_left_over((uint32_t)all, (uint32_t)args.turn) : std::min<int64_t>(args.turn * 3 / 8, all)) * (256 * 256 / (C::BM * C::BN));
    if (tiles == 0) return hipSuccess;
    const TileMap map = MODE == I8Mode::kRows ? TileMap{} : make_tile_map((args.m + HIGH - 1) / HIGH, (args.n + BROAD - 1) / BROAD, (int)all);
    hipLaunchKernelGGL((k_i8_tiles<WM, WN, FM, FN, STAGES, PER_SIMD, MODE, LAST>), dim3((unsigned)tiles), dim3(C::THREADS), C::LDS_BYTES, stream, args, map);
    return hipGetLastError();
}

// The sums of the K ranges, and what the tiles do with a sum.  A thread has 4 columns of a row.
template <I8Mode MODE>
__global__ __launch_bounds__(256) void k_i8_ranges(I8Args p) {
    const int per_row = (p.n + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / per_row;
    if (row >= (MODE == I8Mode::kSums ? (int64_t)p.m * p.groups.groups : p.m)) return;
    const int col = (int)(id - row * per_row) * 4, valid = p.n - col;
    const int32_t *const from = reinterpret_cast<const int32_t *>(p.out.planes) + row * p.out.ldp + col;
    F8Out o = p.out;
    const float *scale_a = p.A.scale + row, *scale_b = p.B.scale + col;
    bool lost = false, nothing = false;
    if constexpr (MODE == I8Mode::kRows) {                     // the last group that begins at the row or before it
        int g = 0;
        for (int step = 1 << 12; step; step /= 2)
            if (g + step < p.groups.groups && i8_span(p.groups, g + step).lo <= row) g += step;
        const I8Span span = i8_span(p.groups, g);
        if (row < span.lo || row >= span.hi) return;
        scale_b += (int64_t)g * p.n;
    } else if constexpr (MODE == I8Mode::kSums) {
        const int64_t g = row / p.m;
        const I8Span span = i8_span(p.groups, (int)g);
        lost = span.hi - span.lo > kI8MaxK;
        nothing = span.hi == span.lo;
        scale_a += g * (p.A.ld_scale - p.m);
        scale_b += g * p.B.ld_scale;
    }
    f8_v4i s{0, 0, 0, 0};
    for (int r0 = 0; r0 < p.ranges; r0 += 4) {                 // four loads at a time: one after the other costs a way to memory each
        f8_v4i x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = *reinterpret_cast<const f8_v4i *>(from + (int64_t)min(r0 + r, p.ranges - 1) * p.out.plane);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r0 + r < p.ranges) s += x[r];
    }
    const int sum[4] = {s[0], s[1], s[2], s[3]};
    if (nothing) {                                             // no infinity or NaN from alpha or from scales
        float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        o.alpha = 0.0f;
        f8_update_row<4>(o, row * o.ldc + col, x, valid);
    } else i8_finish_row<4>(o, row * o.ldc + col, sum, lost ? __builtin_nanf("") : *scale_a, scale_b, valid);
}

// Tiles of 64 x 64 by four wavefronts of 32 x 32, with as many stages as leave all tiles of a call on the device at once, two at least (two | four stages, us: 500 x 300 x 777 7.6 | 6.1; two | three, 640 tiles of
// a gradient with 3 to 6 blocks 17.5 | 11.7); of 64 x 128 with three.  Two teams of wavefronts for alternate blocks of a tile were no faster (500 x 300 x 777 5.5 -> 5.7).
template <I8Mode MODE>
hipError_t launch_form(const I8Args &args, I8Form form, hipStream_t stream) {
    const int64_t tiles = i8_tiles(MODE, form, args);
    if (hipError_t e = form == I8Form::kLarge    ? launch_i8_wide(MODE, args, stream)
                       : form == I8Form::kMiddle ? launch_tiles<2, 2, 2, 4, 3, 2, MODE>(args, form, stream)
                       : tiles <= 512            ? launch_tiles<2, 2, 2, 2, 4, 2, MODE>(args, form, stream)
                       : tiles <= 768            ? launch_tiles<2, 2, 2, 2, 3, 3, MODE>(args, form, stream)
                                                 : launch_tiles<2, 2, 2, 2, 2, 4, MODE>(args, form, stream)) return e;
    if constexpr (MODE != I8Mode::kSums) {
        if (form == I8Form::kLarge && args.ranges == 1) return launch_tiles<2, 2, 2, 4, 3, 2, MODE, true>(args, I8Form::kMiddle, stream);
    }
    if (args.ranges <= 1) return hipSuccess;
    const int64_t threads = (int64_t)args.m * (MODE == I8Mode::kSums ? args.groups.groups : 1) * ((args.n + 3) / 4);
    hipLaunchKernelGGL(k_i8_ranges<MODE>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, args);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_i8_product(I8Mode mode, I8Args args, I8Form form, hipStream_t stream) {
    if (form == I8Form::kThin) return launch_i8_thin(mode, args, stream);
    if (form == I8Form::kLarge) {
        if (hipError_t e = i8_units(&args.turn)) return e;
    }
    if (form == I8Form::kLarge && mode == I8Mode::kSums) {
        if (hipError_t e = launch_i8_wide(mode, args, stream)) return e;
        args.only_short = 1;
        form = I8Form::kMiddle;                              // (half as many workgroups as of 64 x 64, most of which find nothing: 10 -> 5 us for 8 of 4096 x 2048)
    }
    return mode == I8Mode::kDense ? launch_form<I8Mode::kDense>(args, form, stream)
         : mode == I8Mode::kRows  ? launch_form<I8Mode::kRows>(args, form, stream)
                                  : launch_form<I8Mode::kSums>(args, form, stream);
}

}  // namespace oz2
