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
    int ranges, kb_each;                   // kDense: K ranges and their length in blocks
    int only_short;                        // kSums: groups that large tiles take have been served
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
// of 64 x 64 (oz2_i8_gemm.hip) or 256 x 256 (oz2_i8_wide.hip).
enum class I8Form { kThin, kSmall, kLarge };
inline int i8_tile_rows(I8Form form) { return form == I8Form::kThin ? 1 << 30 : form == I8Form::kLarge ? 256 : 64; }
inline int i8_tile_cols(I8Form form) { return form == I8Form::kThin ? 16 : form == I8Form::kLarge ? 256 : 64; }
constexpr int kI8ThinRows = 64;
constexpr int kI8WideBlocks = 3;           // what the kernel of large tiles needs of k, and one whole tile
constexpr int kI8WideGroups = 1024;        // and the most groups that it keeps in LDS
// kSums: groups that it takes; the other ones are left to small tiles.
OZ2_HOST_DEVICE inline bool i8_by_large_tiles(int rows) { return rows > (kI8WideBlocks - 1) * kI8Block && rows <= kI8MaxK; }
// Whether large tiles can serve a call at all.
inline bool i8_large_possible(I8Mode mode, const I8Args &a) {
    return a.m >= 256 && a.n >= 256 && (mode == I8Mode::kDense || a.groups.groups <= kI8WideGroups) && (mode == I8Mode::kSums || i8_blocks(a.k) >= kI8WideBlocks);
}

struct I8Plan {
    I8Form form;
    int ranges, kb_each;                   // K ranges, and blocks of each
    size_t plane_bytes;                    // workspace for the planes of the ranges (0: none needed)
};
inline I8Plan i8_plan(int64_t m, int64_t n, int64_t k) {
    const bool large = m >= 256 && n >= 256 && i8_blocks(k) >= kI8WideBlocks && f8_ceil(m, 256) * f8_ceil(n, 256) >= 64;
    return I8Plan{m <= kI8ThinRows && k > 0 ? I8Form::kThin : large ? I8Form::kLarge : I8Form::kSmall, 1, (int)std::max<int64_t>(i8_blocks(k), 1), 0};
}
// Products by group.
inline I8Form i8_grouped_form(I8Mode mode, const I8Args &a) {
    const int64_t tiles = mode == I8Mode::kRows ? i8_most_units(a.groups.rows, a.groups.groups, 256) : f8_ceil(a.m, 256) * a.groups.groups;
    const int64_t mean = a.groups.rows / a.groups.groups;
    if (mode == I8Mode::kRows && a.k > 0 && mean <= 32) return I8Form::kThin;
    return i8_large_possible(mode, a) && tiles * f8_ceil(a.n, 256) >= 64 && mean >= 256 ? I8Form::kLarge : I8Form::kSmall;
}
inline int64_t i8_plane_ld(int64_t n) { return f8_ceil(n, 16) * 16; }

// Workgroups of a launch.
inline int64_t i8_tiles(I8Mode mode, I8Form form, const I8Args &a) {
    const int64_t tiles_n = f8_ceil(a.n, i8_tile_cols(form));
    if (mode == I8Mode::kRows) return f8_ceil(i8_most_units(a.groups.rows, a.groups.groups, i8_tile_rows(form)) * tiles_n, 8) * 8;
    return f8_ceil(a.m, i8_tile_rows(form)) * tiles_n * (mode == I8Mode::kSums ? a.groups.groups : a.ranges);
}

// Conversions: numbers of a row that 256 threads hold, 8 each and 1, 2, 4 or 8 times.
constexpr int kI8RowThreads = 256, kI8MostHeld = 8 * 8 * kI8RowThreads;
constexpr int kI8ColumnRows = 128, kI8ColumnCols = 512;         // of a workgroup that takes maxima of columns
constexpr int kI8TileThreads = 512;                             // of a tile of 128 x 128 that is turned

// Threads of the largest launch of a conversion.
inline int64_t i8_quantize_units(const I8Groups &g, int64_t each) { return g.offsets ? i8_most_units(g.rows, g.groups, each) : g.groups * f8_ceil(g.each, each); }
inline int64_t i8_quantize_threads(const I8Quantize &p) {
    const int64_t rows = p.groups.rows;
    int64_t most = 0;
    if (p.q) most = p.cols <= 512 ? f8_ceil(rows, 4) * kI8RowThreads : rows * (p.cols <= kI8MostHeld ? kI8RowThreads : 1024);
    if (p.qt) {
        most = std::max(most, f8_ceil(p.side_by_side ? p.cols : p.cols * p.groups.groups, 256) * 256 * (p.side_by_side ? p.groups.groups : 1));
        most = std::max(most, f8_ceil(i8_quantize_units(p.groups, kI8ColumnRows) * f8_ceil(p.cols, kI8ColumnCols), 8) * 8 * 256);
        most = std::max(most, f8_ceil(i8_quantize_units(p.groups, 128) * f8_ceil(p.cols, 128), 8) * 8 * kI8TileThreads);
    }
    return most;
}

#if defined(__HIPCC__)
hipError_t launch_i8_thin(I8Mode mode, const I8Args &args, hipStream_t stream);
hipError_t launch_i8_wide(I8Mode mode, const I8Args &args, hipStream_t stream);
hipError_t launch_i8_product(I8Mode mode, I8Args args, I8Form form, hipStream_t stream);
hipError_t launch_i8_quantize(const I8Quantize &args, int type, hipStream_t stream);
#endif

}  // namespace oz2
