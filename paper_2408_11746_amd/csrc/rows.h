// Rows of numbers as the operators around the products read and write them: four consecutive columns to a lane, fp32, bfloat16 or
// 8 bits, at any alignment that a row of an odd width can have; and the 8-bit form of a group of 128 columns (mst_checkpoint8).
#pragma once

#include "heads.h"

namespace mst {

constexpr int KEPT_GROUP = 128;          // columns that share a unit; 32 lanes have one

// A row of odd width begins in the middle of a 16-byte word.  Global loads and stores of the whole width take any alignment on this
// machine; the types say so to the compiler.
typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short ushort4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t codes4_any __attribute__((aligned(1)));

// n of four columns are there (n >= 4: all); the others are 0, and are not touched in memory.  (Where a row ends inside a quad the last column stands in for
// the missing ones, read or written again: one branch for all of them.)
template <typename T, typename F>
__device__ inline void load_last(const T* p, int n, float (&x)[4], F&& number) {
    x[0] = x[1] = x[2] = x[3] = 0.f;
    if (n > 0) {
        const T a = p[0], b = p[min(1, n - 1)], c = p[min(2, n - 1)];
        x[0] = number(a);
        x[1] = n > 1 ? number(b) : 0.f;
        x[2] = n > 2 ? number(c) : 0.f;
    }
}
template <typename T>
__device__ inline void store_last(T* p, int n, T a, T b, T c) {
    if (n > 0) {
        const T second = n > 1 ? b : a;
        p[0] = a;
        p[min(1, n - 1)] = second;
        p[min(2, n - 1)] = n > 2 ? c : second;
    }
}
__device__ inline void load_columns(const float* p, int n, float (&x)[4]) {
    if (n >= 4) {
        const float4_any v = *reinterpret_cast<const float4_any*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = v[e];
    } else {
        load_last(p, n, x, [](float v) { return v; });
    }
}
__device__ inline void load_columns(const bf16* p, int n, float (&x)[4]) {
    if (n >= 4) {
        const ushort4_any v = *reinterpret_cast<const ushort4_any*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float((uint32_t)v[e] << 16);
    } else {
        load_last(p, n, x, [](bf16 v) { return to_float(v); });
    }
}
__device__ inline void store_columns(float* p, int n, const float (&x)[4]) {
    if (n >= 4) *reinterpret_cast<float4_any*>(p) = float4_any{x[0], x[1], x[2], x[3]};
    else store_last(p, n, x[0], x[1], x[2]);
}
__device__ inline void store_columns(bf16* p, int n, const float (&x)[4]) {
    const uint32_t a = pack2(x[0], x[1]), b = pack2(x[2], x[3]);
    if (n >= 4) *reinterpret_cast<ushort4_any*>(p) = ushort4_any{(unsigned short)a, (unsigned short)(a >> 16), (unsigned short)b, (unsigned short)(b >> 16)};
    else store_last(reinterpret_cast<uint16_t*>(p), n, (uint16_t)a, (uint16_t)(a >> 16), (uint16_t)b);
}
// as the type holds them
__device__ inline void round_columns(const float*, float (&)[4]) {}
__device__ inline void round_columns(const bf16*, float (&x)[4]) {
    const uint32_t a = pack2(x[0], x[1]), b = pack2(x[2], x[3]);
    x[0] = __uint_as_float(a << 16);
    x[1] = __uint_as_float(a & 0xFFFF0000u);
    x[2] = __uint_as_float(b << 16);
    x[3] = __uint_as_float(b & 0xFFFF0000u);
}

// ---- 8 bits: unit = max(top fl(1/127), 2^-126) with top the group's largest size, code = round(v fl(1/unit)), value = code unit.  All steps
// are single fp32 operations, so a group's codes depend on nothing but its numbers.  Sizes are compared as bit patterns, in which no
// number is larger than any: a group with an infinity or no number among its values has such a unit and comes back as no numbers.
constexpr float KEPT_INVERSE = 1.f / 127.f, KEPT_LEAST = 1.17549435e-38f;
__device__ inline float kept_unit(const float (&x)[4]) {       // of the 32 lanes that have the group
    int top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, __float_as_int(x[e]) & 0x7FFFFFFF);
    const float unit = __int_as_float(lanes_max<32>(top)) * KEPT_INVERSE;
    return unit < KEPT_LEAST ? KEPT_LEAST : unit;
}
__device__ inline void store_codes(int8_t* p, int n, const float (&x)[4], float unit) {
#pragma clang fp contract(off)
    const float inverse = 1.f / unit;
    int c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = __float_as_int(x[e] * inverse + 12582912.f);      // 1.5 2^23: the low byte is the nearest whole number (of no number: 0)
    if (n >= 4)
        *reinterpret_cast<codes4_any*>(p) = (uint32_t)(c[0] & 0xFF) | (uint32_t)(c[1] & 0xFF) << 8 | (uint32_t)(c[2] & 0xFF) << 16 | (uint32_t)c[3] << 24;
    else store_last(p, n, (int8_t)c[0], (int8_t)c[1], (int8_t)c[2]);
}
__device__ inline void load_codes(const int8_t* p, int n, float unit, float (&x)[4]) {
    if (n >= 4) {
        const int w = (int)*reinterpret_cast<const codes4_any*>(p);
        x[0] = (float)(w << 24 >> 24) * unit;
        x[1] = (float)(w << 16 >> 24) * unit;
        x[2] = (float)(w << 8 >> 24) * unit;
        x[3] = (float)(w >> 24) * unit;
    } else {
        load_last(p, n, x, [unit](int8_t v) { return (float)v * unit; });
    }
}

inline int check_kept(const mst_checkpoint8* kept) {
    if (!kept->codes_dev || !kept->units_dev || !aligned16(kept->codes_dev) || !aligned16(kept->units_dev)) return MST_ERR_ARG;
    return MST_OK;
}

}  // namespace mst
