// Products of matrices in 8-bit floating point (E4M3, one power of two per block of 128): arguments and launchers of the
// kernels, and the rules by which a call chooses among them.  Everything but the launchers is plain C++ for the CPU tests.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "oz2_tilemap.hpp"

namespace oz2 {

constexpr int kF8Block = 128;              // elements of a row that share a scale

struct F8Matrix {
    const uint8_t *q;                      // E4M3, rows of ld bytes (a multiple of 16)
    int64_t ld;
    const uint8_t *scale;                  // E8M0, rows of ld_scale bytes (a multiple of 4)
    int64_t ld_scale;
    int shift;                             // rows of a block: 2^shift (0 or 7)
};

enum F8Type { kF8Bf16 = 0, kF8F16 = 1, kF8F32 = 2 };
inline int f8_type_bytes(int type) { return type == kF8F32 ? 4 : 2; }

// Where results go: C <- alpha * sum + beta * C; or, gated, H = act(gate) * up in C and, if asked for, the two sums in Z.
struct F8Out {
    void *C;
    int64_t ldc;
    int type;
    float alpha, beta;
    int act;
    void *Z;                               // nullptr: not wanted
    int64_t ldz;
    float *planes;                         // sums of K ranges: [range][m][ldp]; gated: the up part from column ldp / 2 on
    int64_t plane, ldp;
};

struct F8Args {
    F8Matrix A, B;
    int m, n, k;                           // n: columns of C
    int up;                                // gated: row of B where the second weight begins
    int ranges, kb_each;                   // K ranges and their length in blocks (a multiple of 4 if there are several)
    F8Out out;
};

// ------------------------------------------------------------------ which kernel
// kThin: few rows of A, B read once into registers (oz2_f8_thin.hip); the others tiles of C of 64 x 64, 64 x 128 (oz2_f8_gemm.hip) or
// 256 x 256 (oz2_f8_wide.hip), which may cut k into ranges whose sums are added by a second kernel.
enum class F8Form { kThin, kSmall, kMiddle, kLarge };
struct F8Plan {
    F8Form form;
    int ranges, kb_each;                   // K ranges, and blocks of each (a multiple of 4 if there are several)
    size_t plane_bytes;                    // workspace for the planes of the ranges (0: none needed)
    double us;                             // what it is expected to take
};

constexpr int kF8ThinRows = 64;
constexpr int kF8WideBlocks = 3;           // what the kernel of large tiles needs of k, and one whole tile
constexpr int kF8MaxRanges = 16;

inline int64_t f8_blocks(int64_t k) { return (k + kF8Block - 1) / kF8Block; }
inline int64_t f8_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Columns of a plane: those of C, or of both sums; rows of a plane start at multiples of 64 bytes.
inline int64_t f8_plane_ld(int64_t n, bool gated) { return f8_ceil(n, 16) * 16 * (gated ? 2 : 1); }

// Tiles of C (gated: half as wide, since a tile has columns of both weights).
inline int f8_tile_rows(F8Form form) { return form == F8Form::kLarge ? 256 : 64; }
inline int f8_tile_cols(F8Form form) { return form == F8Form::kLarge ? 256 : form == F8Form::kMiddle ? 128 : 64; }
inline int64_t f8_items(F8Form form, int64_t m, int64_t n, bool gated) { return f8_ceil(m, f8_tile_rows(form)) * f8_ceil(n, f8_tile_cols(form) / (gated ? 2 : 1)); }

// What a call takes with tiles of one form, in us: something once, and for each round of the device a time per tile and per block of k.  A
// round is `share` tiles on each of 256 units; in the last one, units with fewer tiles are faster per block.  Fitted to calls of 40
// shapes from 65 x 8192 x 8192 to 4096^3 in a graph, each with all forms and with 1 to 16 ranges; off by 10 % mostly, by a third at most.
// Some, 64 x 64 | 64 x 128 | 256 x 256: 500 x 300 x 777 6.3 | 8.8 | 20; 512 x 4096 x 4096 19 | - | 38; 2048^3 17.6 | 15.4 | 28;
// 3000^3 52 | - | 39; 4096 x 4096 x 512 23 | 24 | 19; 4096^3 105 | - | 60; 8192 x 1024 x 256 10.7 | 12.3 | -; tiles of 128 x 128 were
// behind one of these everywhere.  With ranges: 54 x 205 x 13245 22 (2) -> 9.4 (16), 2048 x 2048 x 16384 103 (one, 64 x 64) -> 74 (4, 256 x 256).
struct F8Cost {
    F8Form form;
    int share;
    double once, per_tile, first_block, further_block;         // per block: the first tile of a unit, each further one
};
constexpr F8Cost kF8Costs[3] = {{F8Form::kSmall, 4, 3.5, 2.2, 0.285, 0.125}, {F8Form::kMiddle, 2, 3.2, 2.8, 0.42, 0.18}, {F8Form::kLarge, 1, 9.0, 3.0, 1.45, 0.0}};
constexpr double kF8LargeFewPerBlock = 1.1;                    // of at most 160 large tiles, which leave units to the others' power and caches
constexpr double kF8RangesOnce = 3.0, kF8PlaneBytesPerUs = 4.0e6;   // the second kernel; planes are written and read
constexpr double kF8BytesPerUs = 5.2e6;                        // from HBM

// The form for few rows: B from HBM, or what a unit's workgroups load through its caches, the rows of A (as a mean of those there are and those of the
// 16, 32 or 64 that the kernel computes) and half of the 16 or 32 of B, for every 16 columns; the unit with the most workgroups counts.  Fitted to 266 calls of 1 to 64
// rows, off by 10 % mostly.
// In us, this form | the best of the others: 1 x 8192 x 8192 13.7 | 16.2; 17 x 8192 x 8192 19.6 | 16.0; 64 x 8192 x 8192 41.6 | 18.1;
// 17 x 4096 x 4096 7.4 | 9.4; 40 x 5120 x 5120 (320 workgroups) 21.6 | 12.2; 33 x 2048 x 2048 6.0 | 7.0; 23 x 84 x 11286 15.3 | 8.5; 60 x 84 x 4000 11.6 | 7.2;
// gated, 16 x 16384 x 4096 28.9 | 34.3; 64 x 16384 x 4096 56.5 | 33.5.
inline double f8_thin_us(int64_t m, int64_t n, int64_t k, bool gated) {
    const double wide = gated ? 2.0 * n : n;
    const int64_t rounds = f8_ceil(f8_ceil(n, 16), 256), computed = m <= 16 ? 16 : m <= 32 ? 32 : 64;
    return std::max(3.0 + rounds * k * ((m + computed) / 2.0 + (gated ? 16 : 8)) / 2.8e4, 1.0 + wide * k / kF8BytesPerUs);
}

inline F8Plan f8_plan(int64_t m, int64_t n, int64_t k, bool gated) {
    const int64_t wide = gated ? 2 * n : n, blocks = f8_blocks(k), groups = f8_ceil(blocks, 4);
    F8Plan best{F8Form::kSmall, 1, (int)std::max<int64_t>(blocks, 1), 0, 1e30};
    if (m <= kF8ThinRows) {
        best.form = F8Form::kThin;
        best.us = f8_thin_us(m, n, k, gated);
    }
    for (const F8Cost &c : kF8Costs) {
        if (c.form == F8Form::kLarge && (m < 256 || wide < 256)) continue;
        const int64_t tiles = f8_items(c.form, m, n, gated), round = 256 * c.share;
        int64_t last = 0;
        for (int64_t asked = 1; asked <= std::min<int64_t>(std::max<int64_t>(groups, 1), kF8MaxRanges); ++asked) {
            const int64_t each = asked == 1 ? std::max<int64_t>(blocks, 1) : f8_ceil(groups, asked) * 4, ranges = std::max<int64_t>(f8_ceil(blocks, each), 1);
            if (ranges == last) continue;
            last = ranges;
            if (c.form == F8Form::kLarge && blocks - (ranges - 1) * each < kF8WideBlocks) continue;
            const int64_t items = tiles * ranges, rounds = items / round, rest = f8_ceil(items - rounds * round, 256);
            const size_t planes = ranges == 1 ? 0 : (size_t)ranges * (size_t)m * (size_t)f8_plane_ld(n, gated) * 4;
            double us = c.once + rounds * (c.per_tile + each * (c.first_block + (c.share - 1) * c.further_block));
            const double first = c.form == F8Form::kLarge && items <= 160 ? kF8LargeFewPerBlock : c.first_block;
            if (rest) us += c.per_tile + each * (first + (rest - 1) * c.further_block);
            us = std::max(us, 3.0 + (double)(m + wide) * k / kF8BytesPerUs) + (planes ? kF8RangesOnce + planes / kF8PlaneBytesPerUs : 0.0);
            if (us < best.us) best = F8Plan{c.form, (int)ranges, (int)each, planes, us};
        }
    }
    return best;
}
// The same without planes.
inline F8Plan f8_plan_one_range(int64_t m, int64_t n, int64_t k, bool gated) {
    F8Plan p = f8_plan(m, n, k, gated);
    p.ranges = 1;
    p.kb_each = (int)std::max<int64_t>(f8_blocks(k), 1);
    p.plane_bytes = 0;
    return p;
}

// ------------------------------------------------------------------ conversions
// Blocks of one row as they are: by rows, unless whole tiles fill the device twice and are nearly all.  Rows | tiles, us, bf16: 1 x 8192 2.2 | 3.2, 1000 x 1111 2.6 | 3.9,
// 140 x 65536 6.0 | 7.0, 1000 x 8191 5.5 | 5.8, 2048 x 4096 5.6 | 4.7, 4096 x 4096 10.5 | 9.2, 16384 x 8192 74 to 79 | 75.
inline bool f8_by_rows(int64_t rows, int64_t cols, bool square, bool transposed) {
    const bool by_tiles = rows / kF8Block * f8_blocks(cols) >= 512 && 8 * (rows / kF8Block) >= 7 * f8_blocks(rows);
    return !square && !transposed && !by_tiles;
}
// Workgroups: by rows 16 blocks of 128 each, otherwise a tile of 128 x 128; of the gated block's gradient one of its two parts, by turns of 8 tiles.
constexpr int kF8RowThreads = 256, kF8TileThreads = 512;
inline int64_t f8_row_groups(int64_t rows, int64_t cols) { return f8_ceil(rows * f8_blocks(cols), 16); }
inline int64_t f8_tile_groups(int64_t rows, int64_t cols) { return f8_blocks(rows) * f8_blocks(cols); }
inline int64_t f8_grad_groups(int64_t m, int64_t f) { return f8_ceil(f8_tile_groups(m, f), 8) * 16; }

#if defined(__HIPCC__)
hipError_t launch_f8_product(const F8Args &args, const F8Plan &plan, bool gated, hipStream_t stream);
hipError_t launch_f8_wide(const F8Args &args, bool gated, hipStream_t stream);
hipError_t launch_f8_thin(const F8Args &args, bool gated, hipStream_t stream);

// What a quantisation writes: either half may be missing (q == nullptr).
struct F8Target {
    uint8_t *q;
    int64_t ld;
    uint8_t *scale;
    int64_t ld_scale;
};
hipError_t launch_f8_quantize(const void *X, int type, int64_t rows, int64_t cols, int64_t ldx, bool square, const F8Target &as_is,
                              const F8Target &transposed, hipStream_t stream);
hipError_t launch_f8_gated_grad(const void *Z, int64_t ldz, const void *dH, int64_t ldh, int type, int64_t m, int64_t f, int64_t up,
                                int act, const F8Target &D, const F8Target &DT, hipStream_t stream);
#endif

}  // namespace oz2
