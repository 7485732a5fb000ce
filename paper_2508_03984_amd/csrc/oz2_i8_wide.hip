// Products of 8-bit integers with a scale for each row on tiles of 256 x 256, by 4 wavefronts of 128 x 128, one per SIMD; the layout of a stage of LDS and the
// arithmetic are those of oz2_i8_gemm.hip.
//
// A matrix instruction takes 16 cycles and a wavefront issues one every 4 or so, so everything else stands between them at an even pace, in the order written.
// Of a block of 128 (64 steps of two instructions, column by column of the 8 x 8 blocks of 16 x 16; a column first with the lower half of the block, so that 8
// instructions lie between two that add to the same accumulators):
//   - all fragments are read from LDS during the block before it: A's into a second set of registers, B's in place, each once its column is
//     done.  So the two stages of LDS (64 KiB each) are free early: A's part of the block after this one from kMeetB on, B's part of
//     this one from kMeetA on.  What is loaded then is the block three (A) and two (B) further on, which has at least 64 steps
//     to arrive.  The loads stand 2 to 4 steps apart, because four wavefronts' take the address unit 64 cycles;
//   - no branch but for what is rare, and scalar work in small pieces;
//   - accumulators are a0 to a255, named in the assembly (as values of the compiler's they were copied and spilled).  Nothing else uses
//     an AGPR or M0, which the tests read from the assembly;
//   - whole tiles of 16-bit results are rounded before the words change places among the lanes.
// A workgroup per compute unit walks over the tiles; its requests run over the ends of tiles.  Every tile has at least kI8WideBlocks blocks.
//
// 8192 x 16384 x 16384 to bf16 1500 to 1550 us, 2.9 POP/s, on numbers of a normal distribution under the power cap (the library's product 1990; the matrix cores from registers 4.1 on random
// operands); 16384 x 8192 x 4096 455, 2.4; 65536 x 4096 x 4096 by 64 experts 1000 to 1030, 2.2.  A block takes 1.4 us, 0.85 of them matrix instructions at the peak clock: LDS is busy three
// quarters of the time (128 KiB of fragments and 64 KiB of loads a block), and the cap holds the clock.  Between two tiles lie about 9 us, for scaling, rounding and 128 KiB of results, which are
// all stored before the next one's sums begin; a group's last tile is half empty on average.  Added to C it is longer: 16 rows of C are asked for, awaited and written before the next ones.  8192 x 8192 x 1024 to bf16 87
// us, added to bf16 152, to f32 106, added to f32 182 (floors 47, 56, 56, 109).
//
// kSums: groups in the order of their lengths and every other round from its end, so that no workgroup has long groups only: 8 groups of 600 to 5800 rows, 4096 x 2048, 184 -> 139 us (8 of 2048: 136).
#include <type_traits>
#include <utility>

#include "oz2_epilogue.hpp"
#include "oz2_i8_device.hpp"

namespace oz2 {
namespace {

typedef __attribute__((address_space(3))) void *lds_ptr_t;

template <typename F, int... I>
__device__ __forceinline__ void static_for_(F &&f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void static_for(F &&f) { static_for_(f, std::make_integer_sequence<int, N>{}); }

extern __shared__ f8_v4i i8_wide_lds[];                       // 2 stages of [256 rows of A | 256 rows of B][128], 1 KiB per wavefront for loads that
                                                              // are not wanted, the scales of the 512 rows, then the groups: kI8WideGroups + 1 first rows, as many numbers of units

constexpr int kStageBytes = 512 * 128, kNowhereAt = 2 * kStageBytes, kScalesAt = kNowhereAt + 4 * 1024, kGroupsAt = kScalesAt + 512 * 4;
constexpr size_t kWideLdsBytes = kGroupsAt + 2 * (kI8WideGroups + 1) * 4;

#define OZ2_TEN(n) "a" #n "0", "a" #n "1", "a" #n "2", "a" #n "3", "a" #n "4", "a" #n "5", "a" #n "6", "a" #n "7", "a" #n "8", "a" #n "9"
__device__ __forceinline__ void claim_accumulators() {
    asm volatile("" ::: "a0", "a1", "a2", "a3", "a4", "a5", "a6", "a7", "a8", "a9", OZ2_TEN(1), OZ2_TEN(2), OZ2_TEN(3), OZ2_TEN(4), OZ2_TEN(5),
                 OZ2_TEN(6), OZ2_TEN(7), OZ2_TEN(8), OZ2_TEN(9), OZ2_TEN(10), OZ2_TEN(11), OZ2_TEN(12), OZ2_TEN(13), OZ2_TEN(14), OZ2_TEN(15),
                 OZ2_TEN(16), OZ2_TEN(17), OZ2_TEN(18), OZ2_TEN(19), OZ2_TEN(20), OZ2_TEN(21), OZ2_TEN(22), OZ2_TEN(23), OZ2_TEN(24), "a250",
                 "a251", "a252", "a253", "a254", "a255");
}
#undef OZ2_TEN

// Accumulator (i, j), the 16 x 16 block of fragments i of A and j of B, is a[32 i + 4 j] to a[32 i + 4 j + 3].
template <int I, int J, bool OPENS>
__device__ __forceinline__ void wide_mfma(const f8_v4i &b, const f8_v4i &a) {
    constexpr int lo = 32 * I + 4 * J, hi = lo + 3;
    if constexpr (OPENS) asm volatile("v_mfma_i32_16x16x64_i8 a[%2:%3], %0, %1, 0" ::"v"(b), "v"(a), "n"(lo), "n"(hi));
    else asm volatile("v_mfma_i32_16x16x64_i8 a[%2:%3], %0, %1, a[%2:%3]" ::"v"(b), "v"(a), "n"(lo), "n"(hi));
}
template <int N>
__device__ __forceinline__ int accumulator() {
    int x;
    asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(x) : "n"(N));
    return x;
}

struct WideArgs {
    I8Args p;
    TileMap map;
    int end;                                                  // kDense, kSums: tiles that are taken
    int tiles_n;                                              // kRows: of a group's
    Divisor by_row, by_band;                                  // by that, and by 8 times that
};
typedef const __attribute__((address_space(4))) WideArgs *ArgsPtr;
// The kernel's arguments where they lie, read anew at each place: kept in registers they were more than there are.
__device__ __forceinline__ ArgsPtr arguments() {
    ArgsPtr a = (ArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(a));
    return a;
}

template <typename T>
__device__ __forceinline__ T fetch(const __attribute__((address_space(4))) T *from) {
    static_assert(sizeof(T) % 4 == 0, "");
    uint32_t words[sizeof(T) / 4];
#pragma unroll
    for (size_t i = 0; i < sizeof(T) / 4; ++i) words[i] = reinterpret_cast<const __attribute__((address_space(4))) uint32_t *>(from)[i];
    T value;
    __builtin_memcpy(&value, words, sizeof value);
    return value;
}

__device__ __forceinline__ const int8_t *uniform(const int8_t *p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
    return reinterpret_cast<const int8_t *>((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Tiles at the edges are moved inwards until they are whole, so that no load needs a bound; of such a tile only what the neighbour does
// not have is stored.  kRows: inwards in all rows that there are, whosesoever.
struct Item {
    int which, row, col, rows;                                // K range or group; first row (kRows: of all) and column, rows that it has (the rest is a neighbour's)
};

template <I8Mode MODE>
struct Wide {
    int lane, wave, lrow, quarter, in_last, cut_kb;
    int a_addr, b_addr;                                       // of a lane's fragments in a stage; the other half is at ^ 64
    int a_offset, b_offset, to_last;                          // a lane's place in the first load of A and of B; what the last block adds
    uint32_t lds0;                                            // where this wavefront's first load goes
    uint32_t a_step, b_step;                                  // 32 rows
    int KB;                                                   // blocks of a row, the last one of which may be cut (kSums: none is)
    uint32_t total;                                           // kRows: tiles
    // What was requested last of either factor: block kb before the end of its tile, rows from these addresses on.
    struct Cursor {
        const int8_t *a, *b;
        int a_kb, a_end, b_kb, b_end;
    } want;
    int a_stage, b_stage;
    // The beginning of the next tile.
    struct Start {
        const int8_t *a, *b;
        int kb, end;
    } follows;

    __device__ __forceinline__ Wide() {
        const ArgsPtr a = arguments();
        lane = threadIdx.x & 63;
        wave = uniform((int)threadIdx.x >> 6);
        lrow = lane & 15;
        quarter = lane >> 4;
        KB = MODE == I8Mode::kSums ? -1 : (a->p.k + kI8Block - 1) / kI8Block;
        in_last = MODE == I8Mode::kSums ? kI8Block : a->p.k - (KB - 1) * kI8Block;
        cut_kb = in_last < kI8Block ? KB - 2 : -1;
        const uint32_t lda = (uint32_t)a->p.A.ld, ldb = (uint32_t)a->p.B.ld;
        a_step = 32 * lda;
        b_step = 32 * ldb;
        const int swizzled = (quarter ^ (lane >> 1 & 7)) * 16;
        a_addr = ((wave >> 1) * 128 + lrow) * 128 + swizzled;
        b_addr = (256 + (wave & 1) * 128 + lrow) * 128 + swizzled;
        const int lane_row = wave * 8 + (lane >> 3), c = (lane & 7) ^ ((wave & 1) * 4 + quarter);
        a_offset = (int)(lane_row * lda) + c * 16;
        b_offset = (int)(lane_row * ldb) + c * 16;
        to_last = (min(c, (in_last - 1) / 16) - c) * 16;
        lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)i8_wide_lds + wave * 1024;
        a_stage = b_stage = 0;
        total = 0;
    }

    static __device__ __forceinline__ int *group_rows() { return reinterpret_cast<int *>(i8_wide_lds) + kGroupsAt / 4; }
    static __device__ __forceinline__ uint32_t *group_units() { return reinterpret_cast<uint32_t *>(group_rows() + kI8WideGroups + 1); }
    // Where the groups' rows begin and how many tile rows there are up to each group's end, by the first wavefront.
    __device__ __forceinline__ void read_groups() {
        const I8Groups s = fetch(&arguments()->p.groups);
        if (wave == 0) {
            uint32_t before = 0;
            for (int g0 = 0; g0 < s.groups; g0 += 64) {
                const int g = g0 + lane;
                I8Span span{0, 0, 0};
                if (g < s.groups) span = i8_span(s, g);
                const uint32_t running = before + i8_running_sum((uint32_t)(span.hi - span.lo + 255) / 256);
                if (g < s.groups) {
                    group_rows()[g] = span.lo;
                    group_units()[g] = running;
                    if (g == s.groups - 1) group_rows()[g + 1] = span.hi;
                }
                before = i8_last(running);
            }
        }
        __syncthreads();
        if constexpr (MODE == I8Mode::kRows) total = (uint32_t)uniform((int)group_units()[s.groups - 1]) * (uint32_t)arguments()->tiles_n;
    }
    // kSums, up to 64 groups: by the number of their rows, the longest first, in place of the numbers of units.
    __device__ __forceinline__ void sort_groups() {
        const int groups = arguments()->p.groups.groups;
        if (wave == 0) {
            const int g = min(lane, groups - 1), length = max(group_rows()[g + 1], group_rows()[g]) - group_rows()[g];
            int rank = 0;
            for (int h = 0; h < min(groups, 64); ++h) {
                const int other = __builtin_amdgcn_readlane(length, h);
                rank += other > length || (other == length && h < g) ? 1 : 0;
            }
            if (groups <= 64) {
                if (lane < groups) group_units()[rank] = (uint32_t)lane;
            } else
                for (int i = lane; i < groups; i += 64) group_units()[i] = (uint32_t)i;
        }
        __syncthreads();
    }
    // i8_span of a group, from there.
    static __device__ __forceinline__ I8Span span_of(int g) {
        const int lo = uniform(group_rows()[g]);
        return I8Span{g, lo, max(uniform(group_rows()[g + 1]), lo)};
    }

    // The work of an id; false if there is none (or, kSums, none that these tiles are for).
    __device__ __forceinline__ bool find(int id, Item &it) const {
        const ArgsPtr a = arguments();
        if constexpr (MODE == I8Mode::kRows) {
            const uint32_t share = (total + 7) / 8, place = (uint32_t)(id & 7) * share + (uint32_t)(id >> 3);
            if ((uint32_t)(id >> 3) >= share - i8_left_over(share, (uint32_t)a->p.turn / 8) || place >= total) return false;
            const uint32_t tiles_n = (uint32_t)a->tiles_n, unit = (uint32_t)divide((int)place, a->by_row.mul, a->by_row.shift);
            const int groups = a->p.groups.groups;
            for (int g0 = 0; g0 < groups; g0 += 64) {
                const int g = min(g0 + lane, groups - 1);
                const uint64_t beyond = __ballot(group_units()[g] > unit);
                if (!beyond) continue;
                const int at = g0 + __builtin_ctzll(beyond);
                const uint32_t first = at ? (uint32_t)uniform((int)group_units()[max(at - 1, 0)]) : 0u, units = (uint32_t)uniform((int)group_units()[at]) - first;
                const uint32_t piece = place - first * tiles_n;            // bands of 8 rows of tiles, column by column
                const uint32_t band = (uint32_t)divide((int)piece, a->by_band.mul, a->by_band.shift), left = piece - band * 8 * tiles_n, high = min(8u, units - band * 8);
                const uint32_t tc = high == 8 ? left >> 3 : left / high, tr = band * 8 + left - tc * high;
                const I8Span span = span_of(at);
                it.which = at;
                it.row = uniform(span.lo + (int)min(tr, units - 1) * 256); // (the minima hold offsets that do not ascend inside)
                it.col = uniform((int)min(tc, tiles_n - 1) * 256);
                it.rows = min(256, span.hi - it.row);
                return true;
            }
            return false;
        } else {
            if (id >= a->end) return false;
            int which, tr, tc, at = id;
            if constexpr (MODE == I8Mode::kSums) {             // every other round from its end, so that a workgroup's tiles of long and short groups even out
                const int turn = (int)gridDim.x, round = id / turn;
                if (round % 2 && (round + 1) * turn <= a->end) at = (2 * round + 1) * turn - 1 - id;
            }
            map_tile_at(&a->map, at, which, tr, tc);
            it.which = uniform(MODE == I8Mode::kSums ? (int)group_units()[which] : which);
            it.row = uniform(tr) * 256;
            it.col = uniform(tc) * 256;
            it.rows = min(256, a->p.m - it.row);
            if constexpr (MODE == I8Mode::kSums) {
                const I8Span span = span_of(it.which);
                return i8_by_large_tiles(span.hi - span.lo);
            }
            return true;
        }
    }
    // The next id from `id` on, in steps of the grid, that has work.
    __device__ __forceinline__ bool find_from(int &id, Item &it) const {
        if constexpr (MODE == I8Mode::kSums) {
            const int end = arguments()->end;
            for (; id < end; id += (int)gridDim.x)
                if (find(id, it)) return true;
            return false;
        } else return find(id, it);
    }

    __device__ __forceinline__ Start start_of(const Item &it) const {
        const ArgsPtr a = arguments();
        const int row0 = min(it.row, a->p.m - 256), col0 = min(it.col, a->p.n - 256);
        Start s;
        int64_t from = 0, b_row = col0;
        s.kb = 0;
        s.end = KB;
        if constexpr (MODE == I8Mode::kDense) {
            s.kb = it.which * a->p.kb_each;
            s.end = min(s.kb + a->p.kb_each, KB);
            from = (int64_t)s.kb * kI8Block;
        } else if constexpr (MODE == I8Mode::kRows) {
            b_row += (int64_t)it.which * a->p.n;
        } else {
            const I8Span span = span_of(it.which);
            from = i8_first_col(span);
            s.end = (span.hi - span.lo + kI8Block - 1) / kI8Block;
        }
        s.a = uniform(a->p.A.q + (int64_t)row0 * a->p.A.ld + from);
        s.b = uniform(a->p.B.q + b_row * a->p.B.ld + from);
        return s;
    }
    // The next block of the tile, or the first one of the next tile.
    __device__ __forceinline__ void advance_a(bool stay) {
        const bool ends = want.a_kb + 1 == want.a_end;
        const int8_t *const a = ends ? follows.a : want.a + kI8Block;
        const int kb = ends ? follows.kb : want.a_kb + 1, end = ends ? follows.end : want.a_end;
        want.a = stay ? want.a : a;
        want.a_kb = stay ? want.a_kb : kb;
        want.a_end = stay ? want.a_end : end;
        a_stage ^= stay ? 0 : 1;
    }
    __device__ __forceinline__ void advance_b() {
        const bool ends = want.b_kb + 1 == want.b_end;
        want.b = ends ? follows.b : want.b + kI8Block;
        want.b_kb = ends ? follows.kb : want.b_kb + 1;
        want.b_end = ends ? follows.end : want.b_end;
        b_stage ^= 1;
    }
    // Load H of the 16 of this wavefront and block: 8 rows, 16 bytes per lane; rows 32 (H % 8) + 8 wave + (0 .. 7) of A or of B in
    // the stage.  `at` is the place of the load before, `to` that of the present one in LDS.
    template <int H>
    __device__ __forceinline__ void load(int &at, uint32_t &to, uint32_t to_step) const {
        constexpr bool of_a = H < 8;
        const int8_t *const base = of_a ? want.a : want.b;
        if constexpr (H % 8 == 0) {
            at = (of_a ? a_offset : b_offset) + ((of_a ? want.a_kb : want.b_kb) == KB - 1 ? to_last : 0);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(at), "s"(base) : "memory");
        } else
            asm volatile("s_mov_b32 m0, %1\n\tv_add_u32 %0, %2, %0\n\tglobal_load_lds_dwordx4 %0, %3" : "+v"(at) : "s"(to), "s"(of_a ? a_step : b_step), "s"(base) : "memory");
        to += to_step;
    }
    __device__ __forceinline__ uint32_t a_to() const { return lds0 + a_stage * kStageBytes; }
    __device__ __forceinline__ uint32_t b_to() const { return lds0 + b_stage * kStageBytes + 8 * 4096; }
    __device__ __forceinline__ void request_a() {
        int at = 0;
        uint32_t to = a_to();
        static_for<8>([&](auto h) { load<decltype(h)::value>(at, to, 4096); });
    }
    __device__ __forceinline__ void request_b() {
        int at = 0;
        uint32_t to = b_to();
        static_for<8>([&](auto h) { load<8 + decltype(h)::value>(at, to, 4096); });
    }

    // The scales of the tile's rows of A and B, a word for each in LDS, where they are when its second block is.  This wavefront's are 128 of either.
    __device__ __forceinline__ void request_scales(const Item &it) const {
        const Place p = place_of(it);
        const float *const from = (wave < 2 ? p.scale_a : p.scale_b) + (wave & 1) * 128 + lane;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t to = lds0 - wave * 1024 + kScalesAt + wave * 512 + half * 256;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from + half * 64) : "memory");
        }
    }
    static __device__ __forceinline__ const float *scales() { return reinterpret_cast<const float *>(i8_wide_lds) + kScalesAt / 4; }

    struct Registers {
        f8_v4i a[2][8][2], b[8][2];
    };
    __device__ __forceinline__ f8_v4i fragment(int addr, int i, int half) const {
        return *reinterpret_cast<const f8_v4i *>(reinterpret_cast<const char *>(i8_wide_lds) + i * 2048 + (addr ^ half * 64));
    }
    // What lies behind k in the last block, of a row of A per thread (0 times what B has there is 0).
    __device__ __forceinline__ void cut(int stage) const {
        const int from = in_last >> 4, r = (int)threadIdx.x, f = r >> 1 & 7;
        int none = 0;
        asm volatile("" : "+v"(none));                         // (zeros of the compiler's own would stand in an AGPR)
        f8_v4i *const row = i8_wide_lds + stage * (kStageBytes / 16) + r * 8;
        row[from ^ f] = f8_keep(row[from ^ f], in_last & 15);
        for (int c = from + 1; c < 8; ++c) row[c ^ f] = f8_v4i{none, none, none, none};
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }

    // Block kb of the tile, whose fragments (but B's last one) are in registers; `stage` has it, the other one the next block.  What is
    // outstanding at either meeting, besides what has to be there: the loads of A and of B that came last (the first block of a tile
    // finds everything there).  The last block's loads of A go nowhere: the next tile reads its first fragments anew and requests
    // then.  Nothing here but what is rare is a branch: one costs as much as an MFMA.
    template <bool OPENS, int SET>
    __device__ __forceinline__ void block(Registers &f, int kb, int kb1, int stage) {
        constexpr int kMeetA = 9, kMeetB = 42;
        static_assert(kMeetA + 2 + 4 * 7 < kMeetB && kMeetB + 1 + 3 * 6 >= 8 * 7, "");
        const int here = stage * kStageBytes, next = kStageBytes - here;
        const int a_next = a_addr + next, b_next = b_addr + next, b_here = b_addr + here;
        const bool last = kb + 1 == kb1;
        int a_at = 0, b_at = 0;
        uint32_t to = 0, step = 4096;
        static_for<64>([&](auto number) {
            constexpr int T = decltype(number)::value, j = T / 8, half = T / 4 % 2, i = T % 4 * 2;
            constexpr int U = T - kMeetB - 1;                              // (columns of B are done by then)
            wide_mfma<i, j, OPENS && half == 0>(f.b[j][half], f.a[SET][i][half]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (T == 0) f.b[7][0] = fragment(b_here, 7, 0);
            if constexpr (T > kMeetA && T < kMeetA + 25 && (T - kMeetA) % 3 == 1) {
                f.a[SET ^ 1][(T - kMeetA) / 3][0] = fragment(a_next, (T - kMeetA) / 3, 0);
                f.a[SET ^ 1][(T - kMeetA) / 3][1] = fragment(a_next, (T - kMeetA) / 3, 1);
            }
            if constexpr (U >= 0 && U < 21 && U % 3 == 0) {
                f.b[U / 3][0] = fragment(b_next, U / 3, 0);
                f.b[U / 3][1] = fragment(b_next, U / 3, 1);
            }
            __builtin_amdgcn_sched_barrier(0);
            wide_mfma<i + 1, j, OPENS && half == 0>(f.b[j][half], f.a[SET][i + 1][half]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (T == 0) f.b[7][1] = fragment(b_here, 7, 1);
            if constexpr (T == 3) advance_b();
            if constexpr (T == 4) to = b_to();
            if constexpr (T == kMeetA) {                                   // A's next block is there, and B's part of this one is free
                if constexpr (OPENS) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                else asm volatile("s_waitcnt vmcnt(16) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                if (__builtin_expect(kb == cut_kb, 0)) cut(stage ^ 1);
            }
            if constexpr (T > kMeetA && T < kMeetA + 33 && (T - kMeetA) % 4 == 2) load<8 + (T - kMeetA) / 4>(b_at, to, 4096);
            if constexpr (T == kMeetB - 6) advance_a(last);
            if constexpr (T == kMeetB - 1) {
                to = last ? lds0 + kNowhereAt : a_to();
                step = last ? 0 : 4096;
            }
            if constexpr (T == kMeetB) {                                   // B's next block is there, and A's part of it is free
                if constexpr (OPENS) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                else asm volatile("s_waitcnt vmcnt(16) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
            if constexpr (U >= 1 && U * 2 / 5 < 8 && (U == 1 || U * 2 / 5 != (U - 1) * 2 / 5)) load<U * 2 / 5>(a_at, to, step);
            __builtin_amdgcn_sched_barrier(0);
        });
    }

    // Accumulators (i, j) to (i, j + 3).
    template <int I, int J>
    static __device__ __forceinline__ void take(int (&x)[16]) {
        static_for<16>([&](auto n) { x[decltype(n)::value] = accumulator<32 * I + 4 * J + decltype(n)::value>(); });
    }
    // 16 columns of a row from four blocks of accumulators: quarter q of the wavefront gets block q's.
    static __device__ __forceinline__ void exchange(float (&x)[16]) {
        float y[16];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t d[4] = {__builtin_bit_cast(uint32_t, x[r]), __builtin_bit_cast(uint32_t, x[4 + r]), __builtin_bit_cast(uint32_t, x[8 + r]),
                                   __builtin_bit_cast(uint32_t, x[12 + r])};
            const exchanged_t e = exchange_quarters(d);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int w = e[q];
                y[4 * q + r] = __builtin_bit_cast(float, w);
            }
        }
#pragma unroll
        for (int n = 0; n < 16; ++n) x[n] = y[n];
    }
    // 16 numbers of 16 bits of a row per lane, from four blocks of accumulators: rounded first, so that half as many words are exchanged.
    template <int TYPE>
    static __device__ __forceinline__ void store_sixteen(uint16_t *to, const float (&x)[16], bool ours) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            lo[b] = F8Number<TYPE>::pack(x[4 * b], x[4 * b + 1]);
            hi[b] = F8Number<TYPE>::pack(x[4 * b + 2], x[4 * b + 3]);
        }
        const exchanged_t l = exchange_quarters(lo), h = exchange_quarters(hi);
        const uint32_t w[8] = {(uint32_t)l[0], (uint32_t)h[0], (uint32_t)l[1], (uint32_t)h[1], (uint32_t)l[2], (uint32_t)h[2], (uint32_t)l[3], (uint32_t)h[3]};
        if (ours) f8_store_words<8>(to, w);
    }

    // Where a tile's results go.
    struct Place {
        int row0, col0;                                       // first row and column that were computed
        int lo, hi;                                           // of the 256 rows those that are the tile's own
        int64_t c_row;                                        // row of C for row0
        const float *scale_a, *scale_b;                       // of the first row and column
    };
    __device__ __forceinline__ Place place_of(const Item &it) const {
        const ArgsPtr a = arguments();
        Place p;
        p.row0 = min(it.row, a->p.m - 256);
        p.col0 = min(it.col, a->p.n - 256);
        p.lo = it.row - p.row0;
        p.hi = p.lo + it.rows;
        p.c_row = p.row0;
        p.scale_a = a->p.A.scale + p.row0;
        p.scale_b = a->p.B.scale + p.col0;
        if constexpr (MODE == I8Mode::kRows) p.scale_b += (int64_t)it.which * a->p.n;
        if constexpr (MODE == I8Mode::kSums) {
            p.c_row += (int64_t)it.which * a->p.m;
            p.scale_a += (int64_t)it.which * a->p.A.ld_scale;
            p.scale_b += (int64_t)it.which * a->p.B.ld_scale;
        }
        return p;
    }
    // The scales of a lane's rows (i) and columns (4 of each j).
    struct Scales {
        float a[8];
        f8_v4f b[8];
    };
    __device__ __forceinline__ void read_scales(Scales &s) const {
        const float *const a = scales() + (wave >> 1) * 128 + lrow, *const b = scales() + 256 + (wave & 1) * 128 + quarter * 4;
#pragma unroll
        for (int i = 0; i < 8; ++i) s.a[i] = a[i * 16];
#pragma unroll
        for (int j = 0; j < 8; ++j) s.b[j] = *reinterpret_cast<const f8_v4f *>(b + j * 16);
    }
    template <int I, int J>
    static __device__ __forceinline__ void take_scaled(const Scales &s, float alpha, float (&x)[16]) {
        int n[16];
        take<I, J>(n);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = (float)n[e] * s.a[I] * s.b[J + e / 4][e % 4];
        if (alpha != 1.0f) {                                   // uniform
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] *= alpha;
        }
    }
    // The results of a tile in 16 bits, C not read.  (Columns that a neighbour has, too, are written twice, the same.)
    template <int TYPE>
    __device__ __forceinline__ void store_16_bits(const F8Out &o, const Place &p) const {
        Scales s;
        read_scales(s);
        const int row = (wave >> 1) * 128 + lrow;
        uint16_t *const c = static_cast<uint16_t *>(o.C) + (p.c_row + row) * o.ldc + p.col0 + (wave & 1) * 128 + quarter * 16;
        static_for<8>([&](auto number) {
            constexpr int i = decltype(number)::value;
            const bool ours = row + i * 16 >= p.lo && row + i * 16 < p.hi;
            float x[16], y[16];
            take_scaled<i, 0>(s, o.alpha, x);
            take_scaled<i, 4>(s, o.alpha, y);
            store_sixteen<TYPE>(c + i * 16 * o.ldc, x, ours);
            store_sixteen<TYPE>(c + i * 16 * o.ldc + 64, y, ours);
            __builtin_amdgcn_sched_barrier(0);
        });
    }
    // In binary32, 4 columns of a row per lane as they lie in the accumulators; or the sums themselves.
    template <bool SCALED>
    __device__ __forceinline__ void store_32_bits(float *to, int64_t ld, const Place &p, float alpha) const {
        Scales s;
        if constexpr (SCALED) read_scales(s);
        const int row = (wave >> 1) * 128 + lrow;
        float *const first = to + (p.c_row + row) * ld + p.col0 + (wave & 1) * 128 + quarter * 4;
        static_for<16>([&](auto number) {
            constexpr int i = decltype(number)::value / 2, j0 = decltype(number)::value % 2 * 4;
            const bool ours = row + i * 16 >= p.lo && row + i * 16 < p.hi;
            float x[16];
            if constexpr (SCALED) take_scaled<i, j0>(s, alpha, x);
            else {
                int n[16];
                take<i, j0>(n);
                __builtin_memcpy(x, n, sizeof x);
            }
            if (ours) {
#pragma unroll
                for (int j = 0; j < 4; ++j) __builtin_memcpy(first + i * 16 * ld + (j0 + j) * 16, x + 4 * j, 16);
            }
        });
    }
    __device__ __forceinline__ void store(const Item &it, void *c, float *planes) const {
        const ArgsPtr a = arguments();
        F8Out o = fetch(&a->p.out);
        o.C = c;                                               // (known to be in global memory, unlike what is fetched)
        o.planes = planes;
        const Place p = place_of(it);
        if (MODE == I8Mode::kDense && o.planes) {
            store_32_bits<false>(o.planes + it.which * o.plane, o.ldp, p, 1.0f);
            return;
        }
        if (o.beta == 0.0f) {
            if (o.type == kF8Bf16) store_16_bits<kF8Bf16>(o, p);
            else if (o.type == kF8F16) store_16_bits<kF8F16>(o, p);
            else store_32_bits<true>(static_cast<float *>(o.C), o.ldc, p, o.alpha);
            return;
        }
        // Added to C, 16 rows at a time; this code exists once.
        const int own_row = (wave >> 1) * 128 + lrow;
        float alpha = o.alpha;
        o.alpha = 1.0f;                                        // (applied with the scales)
#pragma unroll 1
        for (int unit = 0; unit < 16; ++unit) {
            float x[16];
            const int row = own_row + unit / 2 * 16;
            const float *const scale = scales() + 256 + (wave & 1) * 128 + unit % 2 * 64 + quarter * 4;
            int n[16];
            static_for<16>([&](auto number) {
                constexpr int N = decltype(number)::value;
                if (unit == N) take<N / 2, N % 2 * 4>(n);
            });
            const float by = scales()[row];
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = (float)n[e] * by * scale[e / 4 * 16 + e % 4] * alpha;
            exchange(x);
            const int col = p.col0 + (wave & 1) * 128 + (unit % 2 * 4 + quarter) * 16, from = max(it.col - col, 0);
            if (row >= p.lo && row < p.hi && from < 16) f8_update_row<16>(o, (p.c_row + row) * o.ldc + col, x, 16, from);
        }
    }
};

template <I8Mode MODE>
__global__ __launch_bounds__(256, 1) void k_i8_wide(WideArgs args) {
    typedef Wide<MODE> W;
    claim_accumulators();
    W w;
    int id = (int)blockIdx.x, stage = 0;
    if constexpr (MODE != I8Mode::kDense) w.read_groups();
    if constexpr (MODE == I8Mode::kSums) w.sort_groups();
    Item it;
    if (!w.find_from(id, it)) return;
    w.follows = w.start_of(it);
    w.want = {w.follows.a, w.follows.b, w.follows.kb, w.follows.end, w.follows.kb, w.follows.end};
    w.request_a();
    w.request_b();
    w.advance_a(false);
    w.advance_b();
    w.request_a();
    w.request_b();
    typename W::Registers f;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    for (;;) {
        const int kb0 = w.follows.kb, kb1 = w.follows.end;
        id += (int)gridDim.x;
        Item next = it;                                                    // (after the last one: anything that may be loaded)
        const bool more = w.find_from(id, next);
        if (!more) next = it;
        w.follows = w.start_of(next);
        // The first two blocks of the tile are there once all wavefronts have come here.
        asm volatile("s_barrier" ::: "memory");
        static_for<8>([&](auto n) {
            constexpr int i = decltype(n)::value;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f.a[0][i][half] = w.fragment(w.a_addr + stage * kStageBytes, i, half);
                if constexpr (i < 7) f.b[i][half] = w.fragment(w.b_addr + stage * kStageBytes, i, half);
            }
        });
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");    // A's part is free for the third block
        w.advance_a(false);
        w.request_a();
        w.request_scales(it);
        int kb = kb0;
        w.template block<true, 0>(f, kb, kb1, stage);
        stage ^= 1;
        for (;;) {
            if (++kb == kb1) break;
            w.template block<false, 1>(f, kb, kb1, stage);
            stage ^= 1;
            if (++kb == kb1) break;
            w.template block<false, 0>(f, kb, kb1, stage);
            stage ^= 1;
        }
        // The accumulators are complete, and so are this wavefront's loads of the next tile's first two blocks (before any store).
        asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
        w.store(it, args.p.out.C, args.p.out.planes);
        if (!more) break;
        it = next;
    }
}

template <I8Mode MODE>
hipError_t launch(const I8Args &args, hipStream_t stream) {
    static thread_local int attr_device = -1;                // the attribute is per device (set again per thread: harmless)
    int dev = -1;
    if (hipError_t e = hipGetDevice(&dev)) return e;
    if (attr_device != dev) {
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_i8_wide<MODE>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kWideLdsBytes)) return e;
        attr_device = dev;
    }
    const int tiles_n = (args.n + 255) / 256;
    const int64_t tiles = i8_tiles(MODE, I8Form::kLarge, args);
    const TileMap map = MODE == I8Mode::kRows ? TileMap{} : make_tile_map((args.m + 255) / 256, tiles_n, (int)tiles);
    const int end = (int)tiles - (MODE == I8Mode::kDense && args.ranges == 1 ? (int)i8_left_over((uint32_t)tiles, (uint32_t)args.turn) : 0);
    if (end == 0) return hipSuccess;
    hipLaunchKernelGGL(k_i8_wide<MODE>, dim3((unsigned)std::min<int64_t>(MODE == I8Mode::kRows ? tiles : end, args.turn)), dim3(256), kWideLdsBytes, stream,
                       WideArgs{args, map, end, tiles_n, make_divisor(tiles_n), make_divisor(8 * tiles_n)});
    return hipGetLastError();
}

}  // namespace

hipError_t i8_units(int *units) {
    static thread_local int device = -1, found = 0;
    int dev = -1;
    if (hipError_t e = hipGetDevice(&dev)) return e;
    if (device != dev) {
        if (hipError_t e = hipDeviceGetAttribute(&found, hipDeviceAttributeMultiprocessorCount, dev)) return e;
        found = std::max(found / 8 * 8, 8);
        device = dev;
    }
    *units = found;
    return hipSuccess;
}

hipError_t launch_i8_wide(I8Mode mode, const I8Args &args, hipStream_t stream) {
    return mode == I8Mode::kDense ? launch<I8Mode::kDense>(args, stream) : mode == I8Mode::kRows ? launch<I8Mode::kRows>(args, stream) : launch<I8Mode::kSums>(args, stream);
}

}  // namespace oz2
