// Products of E4M3 matrices with a power of two per block of 128 on tiles of 256 x 256, by 4 wavefronts of 128 x 128, one per SIMD;
// the layout of a stage of LDS, the edges and the arithmetic are those of oz2_f8_gemm.hip.
//
// A matrix instruction takes 32 cycles and a wavefront issues one every 4 or so: seven others fit beside it, so everything else
// stands between them at an even pace, in the order written.  Of a block of 128 (64 instructions, column by column of the 8 x 8
// blocks of 16 x 16):
//   - all fragments are read from LDS during the block before it: A's into a second set of registers, B's in place, each once its column is
//     done.  So the two stages of LDS (64 KiB each) are free early: A's part of the block after this one from kMeetB on, B's part of
//     this one from kMeetA on.  What is loaded then is the block three (A) and two (B) further on, which has at least 64 instructions
//     to arrive.  The loads stand 2 to 4 instructions apart, because four wavefronts' take the address unit 64 cycles;
//   - no branch but for what is rare, and scalar work in small pieces: 8192 x 16384 x 4096 on constant operands 440 -> 338 us;
//   - accumulators are a0 to a255, named in the assembly (as values of the compiler's they were copied and spilled).  Nothing else uses
//     an AGPR or M0, which the tests read from the assembly;
//   - whole tiles of 16-bit results are rounded before the words change places among the lanes.
// A workgroup per compute unit walks over the tiles; its requests run over the ends of tiles.  Every tile has at least kF8WideBlocks blocks.
//
// 8192 x 16384 x 16384: 1510 to 1630 us, 2.9 to 2.7 PFLOP/s, on numbers of a normal distribution, at 1.7 to 1.9 GHz under the power cap; on constant operands, which leave the clock at
// 2.2 to 2.3 GHz, 1350 us, 3.26 PFLOP/s; on those with the loads taken out 1085.  By 8 wavefronts of 64 x 128, with a second set of wavefronts instead of the order by
// hand, 1725 (1546).  Bound: the matrix cores are busy 69 % of the cycles, at whatever clock the operands leave (66 % on constants).  The other cycles go to waiting for an
// instruction to issue (41 % of the wavefronts' time), to the loads, of which an L2 miss in six comes late (waits and meetings 15 %), and to what lies between
// two tiles, for which there are no registers beside the next one's sums (8192 x 16384 at k = 4096 420 us, 4096 x 8192 at k = 16384 with as many
// operations 389; gated, 8192 x 8192 x 4096 408, with its sums kept 450).
#include <type_traits>
#include <utility>

#include "oz2_epilogue.hpp"
#include "oz2_f8_device.hpp"

namespace oz2 {
namespace {

typedef __attribute__((address_space(3))) void *lds_ptr_t;

template <typename F, int... I>
__device__ __forceinline__ void static_for_(F &&f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void static_for(F &&f) { static_for_(f, std::make_integer_sequence<int, N>{}); }

extern __shared__ f8_v4i f8_wide_lds[];                       // 2 stages of [256 rows of A | 256 rows of B][128], 2 x 512 words of scales,
                                                              // 1 KiB per wavefront for loads that are not wanted

constexpr int kRows = 512, kStageBytes = kRows * 128, kScalesAt = 2 * kStageBytes, kNowhereAt = kScalesAt + 2 * kRows * 4;
constexpr size_t kWideLdsBytes = kNowhereAt + 4 * 1024;

#define OZ2_TEN(n) "a" #n "0", "a" #n "1", "a" #n "2", "a" #n "3", "a" #n "4", "a" #n "5", "a" #n "6", "a" #n "7", "a" #n "8", "a" #n "9"
__device__ __forceinline__ void claim_accumulators() {
    asm volatile("" ::: "a0", "a1", "a2", "a3", "a4", "a5", "a6", "a7", "a8", "a9", OZ2_TEN(1), OZ2_TEN(2), OZ2_TEN(3), OZ2_TEN(4), OZ2_TEN(5),
                 OZ2_TEN(6), OZ2_TEN(7), OZ2_TEN(8), OZ2_TEN(9), OZ2_TEN(10), OZ2_TEN(11), OZ2_TEN(12), OZ2_TEN(13), OZ2_TEN(14), OZ2_TEN(15),
                 OZ2_TEN(16), OZ2_TEN(17), OZ2_TEN(18), OZ2_TEN(19), OZ2_TEN(20), OZ2_TEN(21), OZ2_TEN(22), OZ2_TEN(23), OZ2_TEN(24), "a250",
                 "a251", "a252", "a253", "a254", "a255");
}
#undef OZ2_TEN

// Accumulator (i, j), the 16 x 16 block of fragments i of A and j of B, is a[32 i + 4 j] to a[32 i + 4 j + 3].  BYTE: which of the four
// scales in a register.
template <int I, int J, bool OPENS, int BYTE>
__device__ __forceinline__ void wide_mfma(const f8_v8i &b, const f8_v8i &a, int sb, int sa) {
    constexpr int lo = 32 * I + 4 * J, hi = lo + 3, s0 = BYTE & 1, s1 = BYTE >> 1;
    if constexpr (OPENS)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 a[%4:%5], %0, %1, 0, %2, %3 op_sel:[%6,%6,0] op_sel_hi:[%7,%7,0]" ::"v"(b), "v"(a), "v"(sb), "v"(sa),
                     "n"(lo), "n"(hi), "n"(s0), "n"(s1));
    else
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 a[%4:%5], %0, %1, a[%4:%5], %2, %3 op_sel:[%6,%6,0] op_sel_hi:[%7,%7,0]" ::"v"(b), "v"(a), "v"(sb),
                     "v"(sa), "n"(lo), "n"(hi), "n"(s0), "n"(s1));
}
template <int N>
__device__ __forceinline__ float accumulator() {
    float x;
    asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(x) : "n"(N));
    return x;
}

struct WideArgs {
    F8Args p;
    TileMap map;
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

__device__ __forceinline__ const uint8_t *uniform(const uint8_t *p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
    return reinterpret_cast<const uint8_t *>((uint64_t)hi << 32 | lo);
}

// Tiles at the edges are moved inwards until they are whole, so that no load needs a bound; of such a tile only what the neighbour does
// not have is stored.
struct Item {
    int range, tr, tc;                                        // K range; place of the tile
};
__device__ __forceinline__ Item find_item(int id) {
    Item it;
    map_tile_at(&arguments()->map, id, it.range, it.tr, it.tc);
    it.range = __builtin_amdgcn_readfirstlane(it.range);
    it.tr = __builtin_amdgcn_readfirstlane(it.tr);
    it.tc = __builtin_amdgcn_readfirstlane(it.tc);
    return it;
}
// Blocks of a K range: [first, end).
__device__ __forceinline__ int first_block(int range) { return range * arguments()->p.kb_each; }
__device__ __forceinline__ int end_block(int range) {
    const ArgsPtr a = arguments();
    return min((range + 1) * a->p.kb_each, (a->p.k + kF8Block - 1) / kF8Block);
}

template <bool GATED>
struct Wide {
    static constexpr int COLS = GATED ? 128 : 256;
    int lane, wave, lrow, quarter, KB, in_last, cut_kb;
    int a_addr, b_addr;                                       // of a lane's fragments in a stage; the other half is at ^ 64
    int a_offset, b_offset, to_last;                          // a lane's place in the first load of A and of B; what the last block adds
    uint32_t lds0;                                            // where this wavefront's first load goes
    uint32_t a_step, b_step;                                  // 32 rows
    const uint8_t *scale_base;                                // of the matrix whose scales this wavefront fetches
    uint32_t scale_ld;
    int scale_shift, scale_up;
    // What was requested last of either factor: block kb before the end of its tile, rows from these addresses on.
    struct Cursor {
        const uint8_t *a, *b, *b2;
        int a_kb, a_end, b_kb, b_end, scale_row;
    } want;
    int a_stage, b_stage, want_scales;
    // The beginning of the next tile.
    struct Start {
        const uint8_t *a, *b, *b2;
        int kb, end, scale_row;
    } follows;

    __device__ __forceinline__ Wide() {
        const ArgsPtr a = arguments();
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        lrow = lane & 15;
        quarter = lane >> 4;
        KB = (a->p.k + kF8Block - 1) / kF8Block;
        in_last = a->p.k - (KB - 1) * kF8Block;
        cut_kb = in_last < kF8Block ? KB - 2 : -1;
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
        lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)f8_wide_lds + wave * 1024;
        scale_base = wave < 2 ? a->p.A.scale : a->p.B.scale;
        scale_ld = (uint32_t)(wave < 2 ? a->p.A.ld_scale : a->p.B.ld_scale);
        scale_shift = wave < 2 ? a->p.A.shift : a->p.B.shift;
        scale_up = GATED && wave >= 2 ? a->p.up : 64;          // rows between this wavefront's two loads of scales
        a_stage = b_stage = want_scales = 0;
    }

    __device__ __forceinline__ Start start_of(const Item &it) const {
        const ArgsPtr a = arguments();
        const int row0 = min(it.tr * 256, a->p.m - 256), col0 = min(it.tc * COLS, a->p.n - COLS);
        Start s;
        s.kb = first_block(it.range);
        s.end = end_block(it.range);
        s.a = uniform(a->p.A.q + (int64_t)row0 * a->p.A.ld + (int64_t)s.kb * kF8Block);
        s.b = uniform(a->p.B.q + (int64_t)col0 * a->p.B.ld + (int64_t)s.kb * kF8Block);
        s.b2 = GATED ? uniform(s.b + (int64_t)a->p.up * a->p.B.ld) : s.b;
        s.scale_row = wave < 2 ? row0 + wave * 128 : col0 + (wave - 2) * (GATED ? 64 : 128);
        return s;
    }
    // The next block of the tile, or the first one of the next tile.
    __device__ __forceinline__ void advance_a(bool stay) {
        const bool ends = want.a_kb + 1 == want.a_end;
        const uint8_t *const a = ends ? follows.a : want.a + kF8Block;
        const int kb = ends ? follows.kb : want.a_kb + 1, end = ends ? follows.end : want.a_end;
        want.a = stay ? want.a : a;
        want.a_kb = stay ? want.a_kb : kb;
        want.a_end = stay ? want.a_end : end;
        a_stage ^= stay ? 0 : 1;
    }
    __device__ __forceinline__ void advance_b() {
        const bool ends = want.b_kb + 1 == want.b_end;
        want.b = ends ? follows.b : want.b + kF8Block;
        want.b2 = ends ? follows.b2 : want.b2 + kF8Block;
        want.scale_row = ends ? follows.scale_row : want.scale_row;
        want.b_kb = ends ? follows.kb : want.b_kb + 1;
        want.b_end = ends ? follows.end : want.b_end;
        b_stage ^= 1;
    }
    // Load H of the 16 of this wavefront and block: 8 rows, 16 bytes per lane; rows 32 (H % 8) + 8 wave + (0 .. 7) of A or of B in
    // the stage, which, gated, are rows of the first and of the second weight by turns of 64.  `at` is the place of the load before,
    // `to` that of the present one in LDS.
    template <int H>
    __device__ __forceinline__ void load(int &at, uint32_t &to, uint32_t to_step) const {
        constexpr bool of_a = H < 8;
        constexpr bool second = GATED && !of_a && H / 2 % 2;
        const uint8_t *const base = of_a ? want.a : second ? want.b2 : want.b;
        // place of the first load, the same again in the other weight, or 32 rows further
        if constexpr (H % 8 == 0) at = (of_a ? a_offset : b_offset) + ((of_a ? want.a_kb : want.b_kb) == KB - 1 ? to_last : 0);
        if constexpr (H % 8 == 0)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(at), "s"(base) : "memory");
        else if constexpr (GATED && (H == 10 || H == 14)) {    // back to the first of these 64 rows, in the second weight
            at -= (int)b_step;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(at), "s"(base) : "memory");
        } else
            asm volatile("s_mov_b32 m0, %1\n\tv_add_u32 %0, %2, %0\n\tglobal_load_lds_dwordx4 %0, %3" : "+v"(at) : "s"(to), "s"(of_a ? a_step : b_step), "s"(base) : "memory");
        to += to_step;
    }
    __device__ __forceinline__ uint32_t a_to() const { return lds0 + a_stage * kStageBytes; }
    __device__ __forceinline__ uint32_t b_to() const { return lds0 + b_stage * kStageBytes + 8 * 4096; }
    // The scales of four blocks from B's one on, a word for each row of the stage; this wavefront's rows 128 wave + 64 half + lane.
    __device__ __forceinline__ void load_scales() {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t row = (uint32_t)((want.scale_row + half * scale_up + lane) >> scale_shift);
            const uint8_t *const from = scale_base + want.b_kb + (uint64_t)row * scale_ld;
            const uint32_t to = lds0 + kScalesAt - wave * 512 + (want_scales * kRows + half * 64) * 4;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "memory");
        }
        want_scales ^= 1;
    }
    __device__ __forceinline__ void request_a() {
        int at = 0;
        uint32_t to = a_to();
        static_for<8>([&](auto h) { load<decltype(h)::value>(at, to, 4096); });
    }
    __device__ __forceinline__ void request_b() {
        int at = 0;
        uint32_t to = b_to();
        static_for<8>([&](auto h) { load<8 + decltype(h)::value>(at, to, 4096); });
        if ((want.b_kb & 3) == 0) load_scales();
    }

    struct Registers {
        f8_v8i a[2][8], b[8];
        int sa[8], sb[8];
    };
    __device__ __forceinline__ f8_v8i fragment(int addr, int i) const {
        const char *const at = reinterpret_cast<const char *>(f8_wide_lds) + i * 2048;
        return f8_join(*reinterpret_cast<const f8_v4i *>(at + addr), *reinterpret_cast<const f8_v4i *>(at + (addr ^ 64)));
    }
    __device__ __forceinline__ int scale(int buffer, int first, int i) const {
        int own_row = lrow;
        asm volatile("" : "+v"(own_row));
        return reinterpret_cast<const int *>(f8_wide_lds)[kScalesAt / 4 + buffer * kRows + first + i * 16 + own_row];
    }
    __device__ __forceinline__ int scale_a(int buffer, int i) const { return scale(buffer, (wave >> 1) * 128, i); }
    __device__ __forceinline__ int scale_b(int buffer, int j) const { return scale(buffer, 256 + (wave & 1) * 128, j); }
    // What lies behind k in the last block, of a row of A or B per thread.
    __device__ __forceinline__ void cut(int stage, int first_row) const {
        const int from = in_last >> 4, r = first_row + (int)threadIdx.x, f = r >> 1 & 7;
        int none = 0;
        asm volatile("" : "+v"(none));                         // (zeros of the compiler's own would stand in an AGPR)
        f8_v4i *const row = f8_wide_lds + stage * (kStageBytes / 16) + r * 8;
        row[from ^ f] = f8_keep(row[from ^ f], in_last & 15);
        for (int c = from + 1; c < 8; ++c) row[c ^ f] = f8_v4i{none, none, none, none};
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }

    // Block kb of the tile, whose fragments (but B's last one) are in registers; `stage` has it, the other one the next block.  What is
    // outstanding at either meeting, besides what has to be there: the loads of A and of B that came last (the first block of a tile
    // finds everything there).  The last block's loads of A go nowhere: the next tile reads its first fragments anew and requests
    // then.  Nothing here but what is rare is a branch: one costs as much as an MFMA.
    template <bool OPENS, int BYTE>
    __device__ __forceinline__ void block(Registers &f, int kb, int kb1, int stage, int &scales) {
        constexpr int SET = BYTE & 1, kMeetA = 9, kMeetB = 42;
        static_assert(kMeetA + 2 + 4 * 7 < kMeetB && kMeetB + 1 + 3 * 6 >= 8 * 7, "");
        const int here = stage * kStageBytes, next = kStageBytes - here;
        const int a_next = a_addr + next, b_next = b_addr + next;
        const bool last = kb + 1 == kb1;
        int a_at = 0, b_at = 0;
        uint32_t to = 0, step = 4096;
        static_for<64>([&](auto number) {
            constexpr int T = decltype(number)::value, j = T / 8, i = T % 8;
            wide_mfma<i, j, OPENS, BYTE>(f.b[j], f.a[SET][i], f.sb[j], f.sa[i]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (T == 0) f.b[7] = fragment(b_addr + here, 7);
            if constexpr (T == 1 && BYTE == 0) f.sb[7] = scale_b(scales, 7);
            if constexpr (T == 3) advance_b();
            if constexpr (T == 4) to = b_to();
            if constexpr (T == kMeetA) {                                   // A's next block is there, and B's part of this one is free
                if constexpr (OPENS) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                else asm volatile("s_waitcnt vmcnt(16) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                if (__builtin_expect(kb == cut_kb, 0)) cut(stage ^ 1, 0);
            }
            if constexpr (T > kMeetA && T < kMeetA + 25 && (T - kMeetA) % 3 == 1) f.a[SET ^ 1][(T - kMeetA) / 3] = fragment(a_next, (T - kMeetA) / 3);
            if constexpr (T > kMeetA && T < kMeetA + 33 && (T - kMeetA) % 4 == 2) load<8 + (T - kMeetA) / 4>(b_at, to, 4096);
            if constexpr (T == kMeetB - 2) {
                if (__builtin_expect((want.b_kb & 3) == 0, 0)) load_scales();
            }
            if constexpr (T == kMeetB - 6) advance_a(last);
            if constexpr (T == kMeetB - 1) {
                to = last ? lds0 + kNowhereAt : a_to();
                step = last ? 0 : 4096;
            }
            if constexpr (T == kMeetB) {                                   // B's next block is there, and A's part of it is free
                if constexpr (OPENS) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                else asm volatile("s_waitcnt vmcnt(16) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                if (__builtin_expect(kb == cut_kb, 0)) cut(stage ^ 1, 256);
                if constexpr (BYTE == 3) scales ^= 1;
            }
            constexpr int U = T - kMeetB - 1;                              // (columns of B are done by then)
            if constexpr (U >= 0 && U < 21 && U % 3 == 0) f.b[U / 3] = fragment(b_next, U / 3);
            if constexpr (BYTE == 3 && U >= 1 && U < 22 && U % 3 == 1) f.sb[U / 3] = scale_b(scales, U / 3);
            if constexpr (U >= 1 && U * 2 / 5 < 8 && (U == 1 || U * 2 / 5 != (U - 1) * 2 / 5)) load<U * 2 / 5>(a_at, to, step);
            if constexpr (BYTE == 3 && j == 7) f.sa[i] = scale_a(scales, i);
            __builtin_amdgcn_sched_barrier(0);
        });
    }

    // Accumulators (i, j) to (i, j + 3).
    template <int I, int J>
    static __device__ __forceinline__ void take(float (&x)[16]) {
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
    static __device__ __forceinline__ void store_sixteen(uint16_t *to, const float (&x)[16]) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            lo[b] = F8Number<TYPE>::pack(x[4 * b], x[4 * b + 1]);
            hi[b] = F8Number<TYPE>::pack(x[4 * b + 2], x[4 * b + 3]);
        }
        const exchanged_t l = exchange_quarters(lo), h = exchange_quarters(hi);
        const uint32_t w[8] = {(uint32_t)l[0], (uint32_t)h[0], (uint32_t)l[1], (uint32_t)h[1], (uint32_t)l[2], (uint32_t)h[2], (uint32_t)l[3], (uint32_t)h[3]};
        f8_store_words<8>(to, w);
    }
    // The results of a tile in 16 bits, C not read.  (Of a tile that was moved inwards, what the neighbour has is written twice, the same.)
    template <int TYPE>
    __device__ __forceinline__ void store_16_bits(const F8Out &o, int64_t row0, int64_t col0, int up) const {
        const int64_t row = row0 + (wave >> 1) * 128 + lrow, col = col0 + (wave & 1) * (COLS / 2) + quarter * 16;
        uint16_t *const c = static_cast<uint16_t *>(o.C) + row * o.ldc + col;
        uint16_t *const z = GATED ? static_cast<uint16_t *>(o.Z) + row * o.ldz + col : nullptr;
        static_for<8>([&](auto number) {
            constexpr int i = decltype(number)::value;
            float x[16], y[16];
            take<i, 0>(x);
            take<i, 4>(y);
            if constexpr (GATED) {
                if (o.Z) {
                    store_sixteen<TYPE>(z + i * 16 * o.ldz, x);
                    store_sixteen<TYPE>(z + i * 16 * o.ldz + up, y);
                }
                f8_gated(x, y, o.act);
                store_sixteen<TYPE>(c + i * 16 * o.ldc, x);
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) { x[e] *= o.alpha; y[e] *= o.alpha; }
                store_sixteen<TYPE>(c + i * 16 * o.ldc, x);
                store_sixteen<TYPE>(c + i * 16 * o.ldc + 64, y);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    }
    // The sums in binary32, 4 columns of a row per lane as they lie in the accumulators; gated, the second weight's `second` further.
    __device__ __forceinline__ void store_sums(float *to, int64_t ld, int64_t row0, int64_t col0, int64_t second, float alpha) const {
        float *const first = to + (row0 + (wave >> 1) * 128 + lrow) * ld + col0 + (wave & 1) * (COLS / 2) + quarter * 4;
        static_for<64>([&](auto number) {
            constexpr int i = decltype(number)::value / 8, j = decltype(number)::value % 8;
            f8_v4f x{accumulator<32 * i + 4 * j>(), accumulator<32 * i + 4 * j + 1>(), accumulator<32 * i + 4 * j + 2>(), accumulator<32 * i + 4 * j + 3>()};
            x *= alpha;
            __builtin_memcpy(first + i * 16 * ld + (GATED ? j % 4 * 16 + (j / 4 ? second : 0) : j * 16), &x, 16);
        });
    }
    __device__ __forceinline__ void store(const Item &it, void *c, void *z, float *planes) const {
        const ArgsPtr a = arguments();
        F8Out o = fetch(&a->p.out);
        o.C = c;                                               // (known to be in global memory, unlike what is fetched)
        o.Z = z;
        o.planes = planes;
        const int m = a->p.m, n = a->p.n, up = a->p.up;
        const int row0 = min(it.tr * 256, m - 256), col0 = min(it.tc * COLS, n - COLS);
        if (o.planes) {
            store_sums(o.planes + it.range * o.plane, o.ldp, row0, col0, o.ldp / 2, 1.0f);
            return;
        }
        if (o.beta == 0.0f && (o.type != kF8F32 || !GATED)) {
            if (o.type == kF8Bf16) store_16_bits<kF8Bf16>(o, row0, col0, up);
            else if (o.type == kF8F16) store_16_bits<kF8F16>(o, row0, col0, up);
            else store_sums(static_cast<float *>(o.C), o.ldc, row0, col0, 0, o.alpha);
            return;
        }
        // Anything else, 16 rows at a time; this code exists once.  One way to memory after the other: 8192 x 8192 x 1024 added to C takes 119 us in
        // bf16 and 166 in f32 (76 and 109 without C); gated, 8192 x 8192 x 4096 in f32 446 us, with its sums kept 588 (396 and 453 in bf16).
        const int first = row0 + (wave >> 1) * 128 + lrow;
#pragma unroll 1
        for (int unit = 0; unit < 16; ++unit) {
            float x[16], u[16];
            static_for<16>([&](auto number) {
                constexpr int N = decltype(number)::value;
                if (unit == N) {
                    if constexpr (!GATED) take<N / 2, N % 2 * 4>(x);
                    else if constexpr (N % 2 == 0) { take<N / 2, 0>(x); take<N / 2, 4>(u); }
                }
            });
            if (GATED && unit % 2) continue;
            const int row = first + unit / 2 * 16;
            const int col = col0 + (wave & 1) * (GATED ? 64 : 128) + ((GATED ? 0 : unit % 2 * 4) + quarter) * 16;
            const int from = max(it.tc * COLS - col, 0);
            const bool ours = row >= it.tr * 256 && from < 16;
            exchange(x);
            if constexpr (!GATED) {
                if (ours) f8_update_row<16>(o, (int64_t)row * o.ldc + col, x, 16, from);
            } else {
                exchange(u);
                if (!ours) continue;
                if (o.Z) {
                    f8_store_row<16>(o.Z, o.type, (int64_t)row * o.ldz + col, x, 16, from);
                    f8_store_row<16>(o.Z, o.type, (int64_t)row * o.ldz + up + col, u, 16, from);
                }
                f8_gated(x, u, o.act);
                f8_store_row<16>(o.C, o.type, (int64_t)row * o.ldc + col, x, 16, from);
            }
        }
    }
};

template <bool GATED>
__global__ __launch_bounds__(256, 1) void k_f8_wide(WideArgs args) {
    typedef Wide<GATED> W;
    claim_accumulators();
    W w;
    int id = (int)blockIdx.x, stage = 0, scales = 0;
    Item it = find_item(id);
    w.follows = w.start_of(it);
    w.want = {w.follows.a, w.follows.b, w.follows.b2, w.follows.kb, w.follows.end, w.follows.kb, w.follows.end, w.follows.scale_row};
    w.request_a();
    w.request_b();
    w.advance_a(false);
    w.advance_b();
    w.request_a();
    w.request_b();
    typename W::Registers f;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    for (;;) {
        const int kb0 = first_block(it.range), kb1 = end_block(it.range);
        id += (int)gridDim.x;
        const bool more = id < arguments()->map.total;
        const Item next = more ? find_item(id) : it;                       // (after the last one: anything that may be loaded)
        w.follows = w.start_of(next);
        // The first two blocks of the tile are there once all wavefronts have come here.
        asm volatile("s_barrier" ::: "memory");
        static_for<8>([&](auto n) {
            constexpr int i = decltype(n)::value;
            f.a[0][i] = w.fragment(w.a_addr + stage * kStageBytes, i);
            f.sa[i] = w.scale_a(scales, i);
            if constexpr (i < 7) {
                f.b[i] = w.fragment(w.b_addr + stage * kStageBytes, i);
                f.sb[i] = w.scale_b(scales, i);
            }
        });
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");    // A's part is free for the third block
        w.advance_a(false);
        w.request_a();
        int kb = kb0;
        w.template block<true, 0>(f, kb, kb1, stage, scales);
        stage ^= 1;
        for (;;) {
            if (++kb == kb1) break;
            w.template block<false, 1>(f, kb, kb1, stage, scales);
            stage ^= 1;
            if (++kb == kb1) break;
            w.template block<false, 2>(f, kb, kb1, stage, scales);
            stage ^= 1;
            if (++kb == kb1) break;
            w.template block<false, 3>(f, kb, kb1, stage, scales);
            stage ^= 1;
            if (++kb == kb1) break;
            w.template block<false, 0>(f, kb, kb1, stage, scales);
            stage ^= 1;
        }
        if (((kb1 - kb0) & 3) != 0) scales ^= 1;                      // (a fourth block has changed it)
        // The accumulators are complete, and so are this wavefront's loads of the next tile's first two blocks (before any store).
        asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
        w.store(it, args.p.out.C, args.p.out.Z, args.p.out.planes);
        if (!more) break;
        it = next;
    }
}

}  // namespace

template <bool GATED>
static hipError_t launch(const F8Args &args, hipStream_t stream) {
    static thread_local int attr_device = -1;                // the attribute is per device (set again per thread: harmless)
    int dev = -1;
    if (hipError_t e = hipGetDevice(&dev)) return e;
    static thread_local int units = 0;                       // compute units of that device, in whole rounds of the XCDs
    if (attr_device != dev) {
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_f8_wide<GATED>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kWideLdsBytes)) return e;
        if (hipError_t e = hipDeviceGetAttribute(&units, hipDeviceAttributeMultiprocessorCount, dev)) return e;
        units = std::max(units / 8 * 8, 8);
        attr_device = dev;
    }
    const int tiles_m = (args.m + 255) / 256, tiles_n = (args.n + Wide<GATED>::COLS - 1) / Wide<GATED>::COLS;
    const TileMap map = make_tile_map(tiles_m, tiles_n, tiles_m * tiles_n * args.ranges);
    hipLaunchKernelGGL(k_f8_wide<GATED>, dim3((unsigned)std::min(map.total, units)), dim3(256), kWideLdsBytes, stream, WideArgs{args, map});
    return hipGetLastError();
}

hipError_t launch_f8_wide(const F8Args &args, bool gated, hipStream_t stream) {
    return gated ? launch<true>(args, stream) : launch<false>(args, stream);
}

}  // namespace oz2
