// Device code shared by the kernels of 8-bit floating-point products.
#pragma once
#include <type_traits>

#include <hip/hip_runtime.h>

#include "oz2_f8.hpp"

namespace oz2 {

typedef int f8_v4i __attribute__((ext_vector_type(4)));
typedef int f8_v8i __attribute__((ext_vector_type(8)));
typedef float f8_v4f __attribute__((ext_vector_type(4)));
typedef __bf16 f8_bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 f8_h2 __attribute__((ext_vector_type(2)));
typedef float f8_f2 __attribute__((ext_vector_type(2)));

// acc + sum over 128 of b * a, scaled by 2^(byte 0 of sb - 127) 2^(byte 0 of sa - 127).  Lane l holds of row l % 16 of either factor
// the 32 elements of quarter l / 16 (in the same order for both) and that row's scale; of the result, row 4 (l / 16) + r of b and
// column l % 16, a row of a.
__device__ __forceinline__ f8_v4f f8_mfma(const f8_v8i &b, const f8_v8i &a, const f8_v4f &acc, int sb, int sa) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, 0, 0, 0, sb, 0, sa);
}
__device__ __forceinline__ f8_v8i f8_join(const f8_v4i &lo, const f8_v4i &hi) {
    return f8_v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}
// The first `valid` (at most 16) of 16 bytes, zeros behind them.
__device__ __forceinline__ f8_v4i f8_keep(f8_v4i v, int valid) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int bytes = valid - 4 * w;
        if (bytes < 4) v[w] = bytes <= 0 ? 0 : v[w] & ((1 << 8 * bytes) - 1);
    }
    return v;
}

// Both activations are g / (1 + exp(-s)): s = g (SiLU), s = 2 sqrt(2 / pi) (g + 0.044715 g^3) (GELU, tanh form, since
// (1 + tanh y) / 2 = 1 / (1 + exp(-2 y))).  Their slope is p + g p (1 - p) s' with p = 1 / (1 + exp(-s)).
// The exponential and the reciprocal are the hardware's, each within 1 or 2 units of the last place; with the rounding of s log2(e) the gate is within
// (4 + |s|) 2^-24 of its value.
constexpr float kGeluScale = 1.5957691216057308f, kGeluCube = 0.044715f, kMinusLog2E = -1.4426950408889634f;
template <int ACT>
__device__ __forceinline__ float f8_gate(float g) {
    const float s = ACT ? kGeluScale * __builtin_fmaf(kGeluCube * g * g, g, g) : g;
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s * kMinusLog2E));
}
template <int ACT>
__device__ __forceinline__ float f8_slope(float g, float p) {
    const float ds = ACT ? kGeluScale * __builtin_fmaf(3.0f * kGeluCube * g, g, 1.0f) : 1.0f, q = p * (1.0f - p);
    if (!ACT) return __builtin_fmaf(g, q, p);
    return q > 0.0f ? __builtin_fmaf(g * q, ds, p) : p;         // p is 0 or 1 (or NaN): the slope's limit, also where s' overflows
}
// x <- act(x) u for several numbers, with one branch for all of them; the two gradients, h act(g) and h u act'(g).
template <int N>
__device__ __forceinline__ void f8_gated(float (&x)[N], const float (&u)[N], int act) {
    if (act) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = x[e] * f8_gate<1>(x[e]) * u[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = x[e] * f8_gate<0>(x[e]) * u[e];
    }
}
template <int ACT, int N>
__device__ __forceinline__ void f8_times_act(const float (&g)[N], const float (&h)[N], float (&x)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = h[e] * (g[e] * f8_gate<ACT>(g[e]));
}
template <int ACT, int N>
__device__ __forceinline__ void f8_times_slope(const float (&g)[N], const float (&u)[N], const float (&h)[N], float (&x)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = h[e] * u[e] * f8_slope<ACT>(g[e], f8_gate<ACT>(g[e]));
}

// Numbers of one type from and to binary32, rounded to nearest even.
template <int TYPE>
struct F8Number;
template <>
struct F8Number<kF8Bf16> {
    typedef uint16_t T;
    static __device__ __forceinline__ float get(T x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
    static __device__ __forceinline__ uint32_t pack(float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f8_f2){x, y}, f8_bf2)); }
};
template <>
struct F8Number<kF8F16> {
    typedef uint16_t T;
    static __device__ __forceinline__ float get(T x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ __forceinline__ uint32_t pack(float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f8_f2){x, y}, f8_h2)); }
};
template <>
struct F8Number<kF8F32> {
    typedef float T;
    static __device__ __forceinline__ float get(T x) { return x; }
};

__device__ __forceinline__ float f8_load(const void *C, int type, int64_t at) {
    return type == kF8Bf16 ? F8Number<kF8Bf16>::get(static_cast<const uint16_t *>(C)[at])
         : type == kF8F16  ? F8Number<kF8F16>::get(static_cast<const uint16_t *>(C)[at])
                           : static_cast<const float *>(C)[at];
}
__device__ __forceinline__ void f8_store(void *C, int type, int64_t at, float x) {
    if (type == kF8Bf16) static_cast<uint16_t *>(C)[at] = (uint16_t)F8Number<kF8Bf16>::pack(x, x);
    else if (type == kF8F16) static_cast<uint16_t *>(C)[at] = (uint16_t)F8Number<kF8F16>::pack(x, x);
    else static_cast<float *>(C)[at] = x;
}

// 2 N 16-bit numbers to wherever they lie.  A store off the multiples of 4 bytes takes the memory system twice as long, so then the first and
// the last number go by themselves and the words between them from their own multiples: 8192 x 8193 x 384 83 -> 60 us.
template <int N>
__device__ __forceinline__ void f8_store_words(uint16_t *to, const uint32_t (&w)[N]) {
    const auto store = [](uint16_t *at, const uint32_t *words, auto count) {
        constexpr int n = decltype(count)::value;
        if constexpr (n > 0) __builtin_memcpy(at, words, 4 * n);
    };
    if ((reinterpret_cast<uintptr_t>(to) & 2) == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) store(to + 2 * i, w + i, std::integral_constant<int, N < 4 ? N : 4>{});
        return;
    }
    uint32_t between[N];
#pragma unroll
    for (int i = 0; i + 1 < N; ++i) between[i] = __builtin_amdgcn_alignbyte(w[i + 1], w[i], 2);
    *to = (uint16_t)w[0];
#pragma unroll
    for (int i = 0; i + 4 < N; i += 4) store(to + 1 + 2 * i, between + i, std::integral_constant<int, 4>{});
    store(to + 1 + 2 * ((N - 1) / 4 * 4), between + (N - 1) / 4 * 4, std::integral_constant<int, (N - 1) % 4>{});
    to[2 * N - 1] = (uint16_t)(w[N - 1] >> 16);
}

// N (a multiple of 4) numbers in a row at C[at], of which those from `from` to `valid` are written.  Whole rows go 16 bytes at a time, on
// whatever multiple of the type's size they lie.
template <int N>
__device__ __forceinline__ void f8_store_row(void *C, int type, int64_t at, const float (&x)[N], int valid, int from = 0) {
    if (valid < N || from > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i >= from && i < valid) f8_store(C, type, at + i, x[i]);
        return;
    }
    if (type == kF8F32) {
        float *const to = static_cast<float *>(C) + at;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const f8_v4f w{x[i], x[i + 1], x[i + 2], x[i + 3]};
            __builtin_memcpy(to + i, &w, 16);
        }
        return;
    }
    uint32_t w[N / 2];
    if (type == kF8Bf16) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = F8Number<kF8Bf16>::pack(x[2 * i], x[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = F8Number<kF8F16>::pack(x[2 * i], x[2 * i + 1]);
    }
    f8_store_words<N / 2>(static_cast<uint16_t *>(C) + at, w);
}

// N numbers in a row from C[at] on, all of which exist, 16 (N = 4, 16-bit: 8) bytes at a time: a product of 8192 x 8192 x 1024 that adds to C
// takes 118 us so, 244 one by one (and 83 without C).
template <int N>
__device__ __forceinline__ void f8_load_row(const void *C, int type, int64_t at, float (&x)[N]) {
    if (type == kF8F32) {
        f8_v4f w[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) __builtin_memcpy(&w[i], static_cast<const float *>(C) + at + 4 * i, 16);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = w[i / 4][i % 4];
        return;
    }
    const uint16_t *const from = static_cast<const uint16_t *>(C) + at;
    uint32_t w[N / 2];
    if constexpr (N == 4) __builtin_memcpy(w, from, 8);
    else {
#pragma unroll
        for (int i = 0; i < N / 2; i += 4) __builtin_memcpy(w + i, from + 2 * i, 16);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint16_t half = (uint16_t)(w[i / 2] >> (i % 2 * 16));
        x[i] = type == kF8Bf16 ? F8Number<kF8Bf16>::get(half) : F8Number<kF8F16>::get(half);
    }
}

// alpha * x + beta * C, and its store; of the row, those from `from` to `valid`.  (What precedes them exists, too.)
template <int N>
__device__ __forceinline__ void f8_update_row(const F8Out &o, int64_t at, float (&x)[N], int valid, int from = 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= o.alpha;
    if (o.beta != 0.0f) {
        float c[N];
        if (valid >= N) f8_load_row<N>(o.C, o.type, at, c);
        else {
#pragma unroll
            for (int i = 0; i < N; ++i) c[i] = f8_load(o.C, o.type, at + min(i, valid - 1));
        }
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __builtin_fmaf(o.beta, c[i], x[i]);
    }
    f8_store_row<N>(o.C, o.type, at, x, valid, from);
}

}  // namespace oz2
