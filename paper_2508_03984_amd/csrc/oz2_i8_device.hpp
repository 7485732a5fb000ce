// Device code shared by the kernels of 8-bit integer products.
#pragma once
#include "oz2_f8_device.hpp"
#include "oz2_i8.hpp"

namespace oz2 {

// Rows lo to hi - 1 of group g, whatever the offsets are.
struct I8Span {
    int group, lo, hi;
};
__device__ __forceinline__ I8Span i8_span(const I8Groups &s, int g) {
    if (!s.offsets) return I8Span{g, g * s.each, (g + 1) * s.each};
    const int lo = min(max(s.offsets[g], 0), s.rows);
    return I8Span{g, lo, min(max(s.offsets[g + 1], lo), s.rows)};
}

// The sums over lanes 0 to l, by moves within rows of 16 lanes, then of the rows' last lanes.
template <int CONTROL, int ROWS>
__device__ __forceinline__ uint32_t i8_plus_moved(uint32_t x) { return x + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, ROWS, 0xf, false); }
__device__ __forceinline__ uint32_t i8_running_sum(uint32_t x) {
    x = i8_plus_moved<0x111, 0xf>(x);                          // from the lane before, 2, 4, 8 before
    x = i8_plus_moved<0x112, 0xf>(x);
    x = i8_plus_moved<0x114, 0xf>(x);
    x = i8_plus_moved<0x118, 0xf>(x);
    x = i8_plus_moved<0x142, 0xa>(x);                          // lane 15 to lanes 16 .. 31, lane 47 to 48 .. 63
    return i8_plus_moved<0x143, 0xc>(x);                       // lane 31 to the upper half
}
__device__ __forceinline__ uint32_t i8_last(uint32_t running) { return (uint32_t)__builtin_amdgcn_readlane((int)running, 63); }

// The groups cut into units of `each` rows, `per` pieces of work to a unit: the piece at the place that `choose` gives for their number (none: -1); false if there is
// none.  A wavefront does this together, 64 groups at a time; piece counts of offsets that do not ascend may be anything, but a span is always one of i8_span's.
struct I8Place {
    I8Span span;
    uint32_t units, piece;                                     // of the group; 0 .. units * per - 1
};
template <typename Choose>
__device__ __forceinline__ bool i8_find_place(const I8Groups &s, int each, uint32_t per, Choose &&choose, I8Place &out) {
    if (!s.offsets) {
        out.units = (uint32_t)(s.each + each - 1) / (uint32_t)each;
        const uint32_t pieces = out.units * per, place = choose(pieces * (uint32_t)s.groups);
        if (place >= pieces * (uint32_t)s.groups) return false;
        const int g = (int)(place / pieces);
        out.span = i8_span(s, g);
        out.piece = place - (uint32_t)g * pieces;
        return true;
    }
    const int lane = threadIdx.x & 63;
    const auto count = [&](int g) {
        if (g >= s.groups) return 0u;
        const I8Span span = i8_span(s, g);
        return (uint32_t)(span.hi - span.lo + each - 1) / (uint32_t)each;
    };
    uint32_t first = count(lane), running = i8_running_sum(first), total = i8_last(running);
    for (int g0 = 64; g0 < s.groups; g0 += 64) total += i8_last(i8_running_sum(count(g0 + lane)));
    total *= per;
    const uint32_t place = choose(total);
    if (place >= total) return false;                          // uniform
    const uint32_t unit = place / per;
    uint32_t before = 0;
    for (int g0 = 0; g0 < s.groups; g0 += 64) {
        if (g0) {
            first = count(g0 + lane);
            running = i8_running_sum(first);
        }
        const uint64_t beyond = __ballot(before + running > unit);
        if (beyond) {
            const int at = __builtin_ctzll(beyond);
            out.span = i8_span(s, __builtin_amdgcn_readfirstlane(g0 + at));
            out.units = (uint32_t)__builtin_amdgcn_readlane((int)first, at);
            out.piece = place - (before + (uint32_t)__builtin_amdgcn_readlane((int)running, at) - out.units) * per;
            out.span.lo = __builtin_amdgcn_readfirstlane(out.span.lo);
            out.span.hi = __builtin_amdgcn_readfirstlane(out.span.hi);
            out.units = (uint32_t)__builtin_amdgcn_readfirstlane((int)out.units);
            out.piece = (uint32_t)__builtin_amdgcn_readfirstlane((int)out.piece);
            return out.piece < out.units * per;
        }
        before += i8_last(running);
    }
    return false;
}
// A workgroup's piece, from its id: each of the 8 XCDs, to which ids go in turns, has neighbouring pieces, which share their operands in its L2.
__device__ __forceinline__ bool i8_find(const I8Groups &s, int each, uint32_t per, uint32_t id, I8Place &out) {
    return i8_find_place(s, each, per, [&](uint32_t total) {
        const uint32_t share = (total + 7) / 8;
        return (id >> 3) < share ? (id & 7) * share + (id >> 3) : ~0u;
    }, out);
}

// First column of a group whose rows lie side by side with the others'.
__device__ __forceinline__ int64_t i8_first_col(const I8Span &s) { return (int64_t)(s.lo / kI8Block + s.group) * kI8Block; }

// Entries of C from sums: N of a row, of which `valid` exist, with the scale of the row and those of the columns.
template <int N>
__device__ __forceinline__ void i8_finish_row(const F8Out &o, int64_t at, const int (&sum)[N], float a, const float *b, int valid) {
    float x[N], scale[N];
    if (valid >= N) __builtin_memcpy(scale, b, sizeof scale);
    else {
#pragma unroll
        for (int i = 0; i < N; ++i) scale[i] = b[min(i, valid - 1)];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)sum[i] * a * scale[i];
    f8_update_row<N>(o, at, x, valid);
}

}  // namespace oz2
