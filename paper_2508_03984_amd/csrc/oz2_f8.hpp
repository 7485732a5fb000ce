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
    int vec;                               // rows of C allow 16-byte accesses at columns that are multiples of 16
    float alpha, beta;
    int act;
    void *Z;                               // nullptr: not wanted
    int64_t ldz;
    int z_vec;
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
enum class F8Form { kThin, kSmall, kLarge };
struct F8Plan {
    F8Form form;
    int ranges, kb_each;
    size_t plane_bytes;                    // workspace for the planes of the ranges (0: none needed)
};

constexpr int kF8ThinRows = 64;
constexpr int kF8WideBlocks = 3;           // what the kernel of large tiles needs of k, and one whole tile
constexpr int kF8MaxRanges = 16;

inline int64_t f8_blocks(int64_t k) { return (k + kF8Block - 1) / kF8Block; }
inline int64_t f8_tiles(int64_t rows, int64_t cols, int tile) { return ((rows + tile - 1) / tile) * ((cols + tile - 1) / tile); }
// Columns of a plane: those of C, or of both sums; rows of a plane start at multiples of 64 bytes.
inline int64_t f8_plane_ld(int64_t n, bool gated) { return (n + 15) / 16 * 16 * (gated ? 2 : 1); }

inline F8Plan f8_plan(int64_t m, int64_t n, int64_t k, bool gated) {
    const int64_t wide = gated ? 2 * n : n, blocks = f8_blocks(k);
    F8Plan p{F8Form::kSmall, 1, (int)std::max<int64_t>(blocks, 1), 0};
    if (m <= kF8ThinRows) {
        p.form = F8Form::kThin;
        return p;
    }
    const int64_t large = f8_tiles(m, wide, 256), small = f8_tiles(m, wide, 128);
    if (large >= 192 && m >= 256 && wide >= 256 && blocks >= kF8WideBlocks) {
        p.form = F8Form::kLarge;
        return p;
    }
    const int64_t groups = (blocks + 3) / 4;               // ranges are whole groups of 4 blocks
    int64_t ranges = std::min<int64_t>({512 / std::max<int64_t>(small, 1), groups / 2, kF8MaxRanges});
    if (ranges > 1) {
        const int64_t each = (groups + ranges - 1) / ranges;
        ranges = (groups + each - 1) / each;               // none empty
        p.ranges = (int)ranges;
        p.kb_each = (int)each * 4;
        p.plane_bytes = (size_t)ranges * (size_t)m * (size_t)f8_plane_ld(n, gated) * 4;
    }
    return p;
}

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
