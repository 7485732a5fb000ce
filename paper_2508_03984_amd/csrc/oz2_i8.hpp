// Products of matrices in 8-bit integers with a scale for each row, alone and grouped by expert: arguments and launchers of the kernels, and the
// rules by which a call chooses among them.  Everything but the launchers is plain C++ for the CPU tests.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "oz2_f8.hpp"

namespace oz2 {

constexpr int kI8Block = 128;              // of k, what a stage of LDS holds of a row; groups that lie side by side start at multiples of it
constexpr int64_t kI8MaxK = 131071;        // 128 * 128 * k stays below 2^31
constexpr int64_t kI8MaxGroups = 4096;

struct I8Matrix {
    const int8_t *q;                       // rows of ld bytes (a multiple of 16)
    int64_t ld;
    const float *scale;                    // of row r in group g: scale[g * ld_scale + r] where rows are cut into groups, else scale[r]
    int64_t ld_scale;
};

// Which rows belong to which group: offsets[g] to offsets[g + 1] - 1, on the device.  Whatever they are, a group is taken as rows lo to hi - 1 with 0 <= lo <= hi <=
// rows.  No offsets: `each` rows for every group (at least one).
struct I8Groups {
    const int32_t *offsets;
    int groups, rows, each;
};

// kDense: C = A B^T.  kRows: rows of A and C by group, with B's rows from g n on.  kSums: the group's columns of A and B, which lie side by side;
// C's rows from g m on.
enum class I8Mode { kDense, kRows, kSums };

struct I8Args {
    I8Matrix A, B;
    int m, n, k;                           // kRows: m = rows of A at most; kSums: k = the most that a group may have
    I8Groups groups;
    int ranges, kb_each;                   // K ranges and their length in blocks (kSums: each group's own)
    int only_short;                        // kSums: groups that large tiles take have been served
    int turn;                              // large tiles of a round (one to a compute unit); kDense, kRows: if a last round is short, tiles of kMiddle take its place
    F8Out out;                             // (planes hold int32 sums)
};

struct I8Quantize {
    const void *X;
    int64_t ldx, x_rows, cols;
    const int32_t *index;                  // row of X for a row of the result, nullptr: the same
    I8Groups groups;
    int8_t *q, *qt;                        // as it is, transposed; nullptr: not wanted
    int64_t ld, ldt;
    float *scale, *scale_t;
    int64_t ld_scale_t;                    // between the groups' scales of the transpose
    int side_by_side;                      // groups of the transpose: side by side, or one below the other
};

inline int64_t i8_blocks(int64_t k) { return f8_ceil(k, kI8Block); }
// Columns of `rows` rows in groups that lie side by side: group g starts at offsets[g] / 128 * 128 + 128 g, and what it needs up to a multiple
// of 128 ends before the next one's start (offsets[g + 1] / 128 * 128 + 128 - offsets[g] / 128 * 128 is more than its rows and a multiple of 128).
inline int64_t i8_grouped_cols(int64_t rows, int64_t groups) { return rows / kI8Block * kI8Block + groups * kI8Block; }

// Units of `each` rows that the rows of all groups have at most, each group's last one counted whole.
inline int64_t i8_most_units(int64_t rows, int64_t groups, int64_t each) { return rows / each + std::min(groups, rows); }

// kThin: few rows (of a group), B read once into registers, 16 columns of C (of a group) to a workgroup (oz2_i8_thin.hip).  The others tiles of C
// of 64 x 64, 64 x 128 (oz2_i8_gemm.hip) or 256 x 256 (oz2_i8_wide.hip), the smaller two, and all of kDense, over ranges of k if there are few, whose sums a second kernel adds.
enum class I8Form { kThin, kSmall, kMiddle, kLarge };
inline int i8_tile_rows(I8Form form) { return form == I8Form::kThin ? 1 << 30 : form == I8Form::kLarge ? 256 : 64; }
inline int i8_tile_cols(I8Form form) { return form == I8Form::kThin ? 16 : form == I8Form::kLarge ? 256 : form == I8Form::kMiddle ? 128 : 64; }
constexpr int kI8ThinRows = 64;
constexpr int kI8WideBlocks = 3;           // what the kernel of large tiles needs of k, and one whole tile
constexpr int kI8WideGroups = 1024;        // and the most groups that it keeps in LDS
// kSums: groups that it takes; the other ones are left to small tiles.
OZ2_HOST_DEVICE inline bool i8_by_large_tiles(int rows) { return rows > (kI8WideBlocks - 1) * kI8Block && rows <= kI8MaxK; }
// Of `share` large tiles, `turn` of which go at a time, those that are left to tiles of 64 x 128 (8 for a large one): the ones of a last round, not the only one, that has at
// most 3 / 8 of its places filled.  kRows counts by XCD.  16384 x 2048 x 4096 in 8 groups of 500 to 4000 rows, 560 tiles: 148 -> 122 us; one group, 512 tiles, 110.
OZ2_HOST_DEVICE inline uint32_t i8_left_over(uint32_t share, uint32_t turn) {
    const uint32_t rest = share % turn;
    return share > turn && rest <= turn * 3 / 8 ? rest : 0;
}
// Whether large tiles can serve a call at all.
inline bool i8_large_possible(I8Mode mode, const I8Args &a) {
    return a.m >= 256 && a.n >= 256 && (mode == I8Mode::kDense || a.groups.groups <= kI8WideGroups) && (mode == I8Mode::kSums || i8_blocks(a.k) >= kI8WideBlocks);
}

struct I8Plan {
    I8Form form;
    int ranges, kb_each;                   // K ranges, and blocks of each (kSums: 0)
    size_t plane_bytes;                    // workspace for the planes of the ranges (0: none needed)
    double us;                             // what it is expected to take
};
inline int64_t i8_plane_ld(int64_t n) { return f8_ceil(n, 16) * 16; }

// What a call takes with tiles of one form, in us: something once, and for each round of the device a time per tile and per block of k; a round is `share` tiles on each of
// 256 units, in the last one units with fewer tiles are faster per block.  Measured, 64 x 64 | 64 x 128 | 256 x 256: 500 x 300 x 777 5.7 | 8.3 | 16; 1024 x 4096 x 4096 27.7 | 23.4 | 44; 2048^3
// 15.6 | 13.2 | 26; 3000^3 51 | 46 | 38; 4096 x 4096 x 512 20.4 | 21.5 | 19.2; 8192 x 1024 x 256 9.4 | 10.1 | -.  With ranges: 100 x 100 x 20000 42 -> 9.3 (16), 512 x 512 x 4096 11.0 -> 10.1 (3), 1536 x 1000 x 40000
// 342 -> 69 (10, of large tiles).  Of 36 shapes the choice is within 3 % of the best of all forms and ranges, 8 % at worst (65 x 8192 x 8192 22.1 | 20.5).
struct I8Cost {
    I8Form form;
    int share;
    double once, per_tile, first_block, further_block;         // per block: the first tile of a unit, each further one
};
constexpr I8Cost kI8Costs[3] = {{I8Form::kSmall, 4, 3.5, 2.2, 0.285, 0.125}, {I8Form::kMiddle, 2, 3.2, 2.8, 0.42, 0.18}, {I8Form::kLarge, 1, 9.0, 3.0, 1.45, 0.0}};
constexpr double kI8RangesOnce = 3.0, kI8PlaneBytesPerUs = 4.0e6;   // the second kernel; planes are written and read
constexpr double kI8BytesPerUs = 5.2e6;                        // from HBM
constexpr int kI8MaxRanges = 16;

// The form for few rows: B from HBM, or what a unit's workgroups load through its caches.  This form | the best of the others: 1 x 8192 x 8192 13.9 | 16; 33 x 2048 x 2048 5.9 | 6.8; 17 x 8192 x 8192 19.5 | 15.0;
// 64 x 8192 x 8192 41 | 17.4; 16 x 128 x 16384 16.3 | 8.3; 8 x 300 x 700 3.1 | 5.2.
inline double i8_thin_us(int64_t m, int64_t n, int64_t k) {
    const int64_t rounds = f8_ceil(f8_ceil(n, 16), 256), computed = m <= 16 ? 16 : m <= 32 ? 32 : 64;
    return std::max(3.0 + rounds * k * ((m + computed) / 2.0 + 8) / 2.8e4, 1.0 + (double)n * k / kI8BytesPerUs);
}

inline I8Plan i8_plan(int64_t m, int64_t n, int64_t k) {
    const int64_t blocks = i8_blocks(k);
    I8Plan best{I8Form::kSmall, 1, (int)std::max<int64_t>(blocks, 1), 0, 1e30};
    if (m <= kI8ThinRows && k > 0) {
        best.form = I8Form::kThin;
        best.us = i8_thin_us(m, n, k);
    }
    for (const I8Cost &c : kI8Costs) {
        if (c.form == I8Form::kLarge && (m < 256 || n < 256)) continue;
        const int64_t tiles = f8_ceil(m, i8_tile_rows(c.form)) * f8_ceil(n, i8_tile_cols(c.form)), round = 256 * c.share;
        int64_t last = 0;
        for (int64_t asked = 1; asked <= std::min<int64_t>(std::max<int64_t>(blocks, 1), kI8MaxRanges); ++asked) {
            const int64_t each = std::max<int64_t>(f8_ceil(blocks, asked), 1), ranges = std::max<int64_t>(f8_ceil(blocks, each), 1);
            if (ranges == last) continue;
            last = ranges;
            if (c.form == I8Form::kLarge && blocks - (ranges - 1) * each < kI8WideBlocks) continue;
            const int64_t items = tiles * ranges, rounds = items / round, rest = f8_ceil(items - rounds * round, 256);
            const size_t planes = ranges == 1 ? 0 : (size_t)ranges * (size_t)m * (size_t)i8_plane_ld(n) * 4;
            double us = c.once + rounds * (c.per_tile + each * (c.first_block + (c.share - 1) * c.further_block));
            if (c.form == I8Form::kLarge && ranges == 1 && i8_left_over((uint32_t)tiles, 256))
                us += 3.0 + f8_ceil((items - rounds * round) * 8, 512) * (kI8Costs[1].per_tile + each * (kI8Costs[1].first_block + kI8Costs[1].further_block));
            else if (rest) us += c.per_tile + each * (c.first_block + (rest - 1) * c.further_block);
            us = std::max(us, 3.0 + (double)(m + n) * k / kI8BytesPerUs) + (planes ? kI8RangesOnce + planes / kI8PlaneBytesPerUs : 0.0);
            if (us < best.us) best = I8Plan{c.form, (int)ranges, (int)each, planes, us};
        }
    }
    return best;
}
// The same without planes.
inline I8Plan i8_plan_one_range(int64_t m, int64_t n, int64_t k) {
    I8Plan p = i8_plan(m, n, k);
    p.ranges = 1;
    p.kb_each = (int)std::max<int64_t>(i8_blocks(k), 1);
    p.plane_bytes = 0;
    return p;
}
// Products by group, from the mean of their rows, by the costs of single ones (us; small | middle | large): kRows, 64 groups, 2048 x 2048, mean 24 51 | 44 | 67, 64 68 | 56 | 69, 256 160 | 132 | 102;
// 8 groups, 2048 x 1024, mean 100 6.8 | 7.2 | 17, 800 30 | 30 | 23; 8 groups, 8192 x 4096, mean 256 147 | 122 | 100.  kSums, 8 groups, 4096 x 2048, mean 400 74 | 72 | 82, 800
// 112 | 102 | 95, 2000 214 | 190 | 142; 16 groups, 256 x 512, mean 800 9.2 | 11.3 | 32.
// The host does not know who has how many rows, so one long group among short ones goes by the form of the mean: 64 groups, 4096 x 2048, 127 rows (the form for few rows, which reads a group's weight again for every
// 16 rows), 2 each 111 us, one of 64 and 63 of 1 154.
// Few tiles and a long contraction go by ranges of k, too (kSums: as many for every group, of its own blocks), us without | with: kSums, 2 groups of 32768 rows, 100 x 100 68 | 12;
// one of 16384, 1000 x 1000 53 | 36; kRows, 3 groups of 40, 64 x 8192 18.9 | 8.5.  Near the border they lose a little (8 groups of 64, 512 x 4096 11.2 | 13.2), hence 1.2.
inline I8Plan i8_grouped_plan(I8Mode mode, const I8Args &a) {
    const int64_t rows = a.groups.rows, groups = a.groups.groups, mean = rows / groups, sought = std::min(groups, rows);
    const int64_t blocks = mode == I8Mode::kRows ? i8_blocks(a.k) : i8_blocks(mean);
    I8Plan best{I8Form::kThin, 1, (int)std::max<int64_t>(i8_blocks(a.k), 1), 0, 1e30};
    // Thin | small: 64 groups, 4096 x 2048, 1 row 3.9 | 7.0, 32 rows 29 | 29, 256 rows 102 | 88; 4 groups, 512 x 512, 32 rows 3.1 | 4.1; 8 groups, 8192 x 4096, 8 rows 33 | 25.
    if (mode == I8Mode::kRows && a.k > 0 && (mean < 2 || (mean <= 8 && groups * a.n * (int64_t)a.k <= 1 << 21))) return best;
    for (const I8Cost &c : kI8Costs) {
        if (c.form == I8Form::kLarge && (!i8_large_possible(mode, a) || mean < (mode == I8Mode::kRows ? 64 : 768))) continue;
        const int high = i8_tile_rows(c.form);
        const int64_t units = mode == I8Mode::kRows ? std::max(f8_ceil(2 * rows + sought * high, 2 * high), sought) : f8_ceil(a.m, high) * groups;
        const int64_t tiles = units * f8_ceil(a.n, i8_tile_cols(c.form)), round = 256 * c.share;
        const int64_t most = c.form == I8Form::kLarge || tiles > 256 ? 1 : std::min<int64_t>(std::max<int64_t>(blocks / 2, 1), kI8MaxRanges);
        int64_t last = 0;
        for (int64_t asked = 1; asked <= most; ++asked) {
            const int64_t each = std::max<int64_t>(f8_ceil(blocks, asked), 1), ranges = std::max<int64_t>(f8_ceil(blocks, each), 1);
            if (ranges == last) continue;
            last = ranges;
            const int64_t items = tiles * ranges, rounds = items / round, rest = f8_ceil(items - rounds * round, 256);
            const size_t planes = ranges == 1 ? 0 : (size_t)ranges * (size_t)(mode == I8Mode::kRows ? rows : groups * a.m) * (size_t)i8_plane_ld(a.n) * 4;
            const double whole = c.per_tile + each * (c.first_block + (c.share - 1) * c.further_block);
            double us = c.once + rounds * whole;
            if (rest) us += c.per_tile + each * (c.first_block + (rest - 1) * c.further_block);
            // (by rows the number of tiles is an estimate, and what units share of a weight is read more often)
            if (mode == I8Mode::kRows && rounds == 0 && c.form == I8Form::kMiddle) us *= 1.12;
            if (mode == I8Mode::kRows && rounds > 0) us = c.once + (c.form == I8Form::kSmall ? 1.35 : c.form == I8Form::kMiddle ? 1.2 : 1.08) * ((double)items / round + 0.3) * whole;
            if (planes) us = 1.2 * (us + kI8RangesOnce + planes / kI8PlaneBytesPerUs);
            if (us < best.us) best = I8Plan{c.form, (int)ranges, mode == I8Mode::kRows ? (int)each : 0, planes, us};
        }
    }
    return best;
}
// The same without planes.
inline I8Plan i8_grouped_plan_one_range(I8Mode mode, const I8Args &a) {
    I8Plan p = i8_grouped_plan(mode, a);
    p.ranges = 1;
    p.kb_each = (int)std::max<int64_t>(i8_blocks(a.k), 1);
    p.plane_bytes = 0;
    return p;
}
// Workgroups of a launch.
inline int64_t i8_tiles(I8Mode mode, I8Form form, const I8Args &a) {
    const int64_t tiles_n = f8_ceil(a.n, i8_tile_cols(form)), ranges = std::max(a.ranges, 1);
    if (mode == I8Mode::kRows) return f8_ceil(i8_most_units(a.groups.rows, a.groups.groups, i8_tile_rows(form)) * tiles_n, 8) * 8 * ranges;
    return f8_ceil(a.m, i8_tile_rows(form)) * tiles_n * (mode == I8Mode::kSums ? a.groups.groups : 1) * ranges;
}

// Conversions: numbers of a row that 256 threads hold, 8 each and 1, 2, 4 or 8 times.
constexpr int kI8RowThreads = 256, kI8MostHeld = 8 * 8 * kI8RowThreads;
constexpr int kI8ColumnThreads = 512;                           // of a workgroup that takes maxima of columns
constexpr int kI8TileThreads = 512;                             // of a tile of 128 x 128 that is turned
// Workgroups for the rows of all groups in units of `each`, `parts` to a unit.
inline int64_t i8_quantize_pieces(const I8Groups &g, int64_t each, int64_t parts) {
    return f8_ceil((g.offsets ? i8_most_units(g.rows, g.groups, each) : g.groups * f8_ceil(g.each, each)) * parts, 8) * 8;
}

// lanes: threads to a row that is held (0: it is read twice); rows_each: rows of a workgroup that converts them and takes the maxima of columns with them, 0: it
// takes none; columns_each: rows of one that takes maxima of columns only, 0: there is none; strips: the transpose in one launch, and
// what is written as it is, too, of up to kI8StripCols columns.
struct I8ConvertPlan {
    int lanes, rows_each, columns_each;
    bool strips;
};
constexpr int kI8StripCols = 2048;
inline I8ConvertPlan i8_convert_plan(const I8Quantize &p) {
    const int64_t rows = p.groups.rows, groups = p.groups.groups;
    I8ConvertPlan plan{p.cols <= 32 ? 4 : p.cols <= 128 ? 16 : p.cols <= 512 ? 64 : p.cols <= kI8MostHeld ? 256 : 0, 0, 0, false};
    if (p.cols > 2048 && plan.lanes && rows <= 512) plan.lanes = 1024;    // (a row's numbers spread wider: 64 x 8192 bf16 4.5 -> 3.1 us)
    if (!p.qt) return plan;
    // Few rows to a group (by group the mean says less): one launch.  Three or four | one, us, both forms: 100 x 100 bf16 10.5 | 4.5, 512 x 4096 15.7 | 13.3, 64 of 128 x 512
    // 15.5 | 9.4, 1000 x 1000 15.1 | 16.9, 4000 x 64 12.2 | 37.7.  A long group among short ones is read by a workgroup for every 32 columns all the same: 64 groups, 800 columns, 4630 rows, about 72 each 13.4, one
    // of 4000 and 63 of 10 63.
    if (rows <= (p.groups.offsets ? 384 : 512) * groups && rows * p.cols <= 1 << 22) {
        plan.strips = true;
        return plan;
    }
    // Atomic maxima of one scale take about 20 ns each, one after the other, so at most 128 workgroups raise the same ones (1024 did: 16384 x 512 bf16 22 us, now 7).
    // With the rows (one read less) where that leaves workgroups enough for the device, or little work in all.  Together | apart, us: 8 of 4096 x 2048 f32 126 | 152,
    // 200 x 400 f32 10.1 | 14.0; 4096 x 4096 bf16 50 | 35, 16384 x 4096 150 | 96.
    const int64_t subs = plan.lanes ? kI8RowThreads / std::min(plan.lanes, kI8RowThreads) : 1;
    const bool fused = p.q && plan.lanes && plan.lanes <= kI8RowThreads && (groups >= 6 || rows <= 512);
    const auto whole = [](int64_t each, int64_t of) { return (int)(f8_ceil(std::max<int64_t>(each, 1), of) * of); };
    if (fused) plan.rows_each = whole(std::max(f8_ceil(rows, 128 * groups), f8_ceil(rows, 1024)), subs);
    else {
        const int64_t lanes = p.cols <= 32 ? 4 : p.cols <= 128 ? 16 : 64, parts = f8_ceil(p.cols, lanes * 8);
        plan.columns_each = whole(std::max(f8_ceil(rows, 128 * groups), f8_ceil(rows * parts, 1024)), 4 * kI8ColumnThreads / lanes);
    }
    return plan;
}
// Threads of the largest launch.
inline int64_t i8_quantize_threads(const I8Quantize &p) {
    const I8ConvertPlan plan = i8_convert_plan(p);
    const int64_t rows = p.groups.rows;
    int64_t most = 0;
    if (p.q)
        most = plan.rows_each ? i8_quantize_pieces(p.groups, plan.rows_each, 1) * kI8RowThreads
               : plan.lanes   ? f8_ceil(rows * plan.lanes, kI8RowThreads) * kI8RowThreads
                              : rows * 1024;
    if (plan.strips) most = std::max(most, (f8_ceil(p.cols, 32) * p.groups.groups + f8_ceil(rows, 4)) * 256);
    else if (p.qt) {
        most = std::max(most, f8_ceil(p.side_by_side ? p.cols : p.cols * p.groups.groups, 256) * 256 * (p.side_by_side ? p.groups.groups : 1));
        if (plan.columns_each) most = std::max(most, i8_quantize_pieces(p.groups, plan.columns_each, f8_ceil(p.cols, p.cols <= 32 ? 32 : p.cols <= 128 ? 128 : 512)) * kI8ColumnThreads);
        most = std::max(most, i8_quantize_pieces(p.groups, 128, f8_ceil(p.cols, 128)) * kI8TileThreads);
    }
    return most;
}

#if defined(__HIPCC__)
hipError_t launch_i8_thin(I8Mode mode, const I8Args &args, hipStream_t stream);
hipError_t launch_i8_wide(I8Mode mode, const I8Args &args, hipStream_t stream);
hipError_t i8_units(int *units);              // compute units of the current device, in whole rounds of the XCDs
hipError_t launch_i8_product(I8Mode mode, I8Args args, I8Form form, hipStream_t stream);   // args.ranges, kb_each and out.planes as planned
hipError_t launch_i8_quantize(const I8Quantize &args, int type, hipStream_t stream);
#endif

}  // namespace oz2
