// Heads of queries, keys and values as the attention half of a block reads and writes them: strided views of vectors of
// head_dim contiguous components, their checks on the host, 16-byte loads and the operands of the matrix instructions.
#pragma once

#include "common.h"
#include "split_bf16.h"

namespace mst {

constexpr int HEAD_DIM_MAX = 128;        // of the attention; head_dim is a multiple of 8
constexpr int SELECT_MAX = 64;           // blocks a query may select: one bit each in a word
constexpr int KEY_BLOCKS_MAX = 2048;     // blocks of a sequence: their bit words for 256 queries are 64 KB of LDS
constexpr int64_t HEADS_MAX = 1 << 16;

template <typename T>
struct Heads {                           // element strides of [batch][token][head][head_dim]
    T* p;
    int64_t sb, st, sh;
    __device__ T* at(int b, int64_t t, int h) const { return p + b * sb + t * st + h * sh; }
};

template <typename T>
inline Heads<T> heads_of(const mst_heads* v) {
    return {static_cast<T*>(v->data), v->batch, v->token, v->head};
}

// a view of b x t x h vectors: 16-byte words everywhere, so that a lane loads eight components at once
inline int check_heads(const mst_heads* v, int64_t b, int64_t t, int64_t h, mst_dtype type, bool written) {
    if (!v) return MST_ERR_ARG;
    if (b * t * h == 0) return MST_OK;
    if (!v->data || !aligned16(v->data)) return MST_ERR_ARG;
    const int64_t word = type == MST_F32 ? 4 : 8;
    const int64_t n[3] = {b, t, h}, s[3] = {v->batch, v->token, v->head};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (s[i] < 0 || s[i] % word != 0 || (written && s[i] == 0) || s[i] > (int64_t(1) << 40))) return MST_ERR_ARG;
    return MST_OK;
}

inline bool is_type(mst_dtype t) { return t == MST_F32 || t == MST_BF16; }

struct bf16 { uint16_t bits; };          // storage of a bfloat16

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }

// eight consecutive components as fp32 (one 16-byte load, or two)
__device__ inline void load8(const float* p, float (&x)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ inline void load8(const bf16* p, float (&x)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ inline void store8(float* p, const float (&x)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ inline void store8(bf16* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(cvt_pk_bf16(x[0], x[1]), cvt_pk_bf16(x[2], x[3]), cvt_pk_bf16(x[4], x[5]), cvt_pk_bf16(x[6], x[7]));
}
__device__ inline void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ inline void store4(bf16* p, float a, float b, float c, float d) {
    *reinterpret_cast<uint2*>(p) = make_uint2(cvt_pk_bf16(a, b), cvt_pk_bf16(c, d));
}

// ---- operands of a 16 x 16 x 32 product.  Lane l holds row (or column) l % 16 and the eight contraction indices of lane
// group l / 16.  Which eight is free as long as both operands agree: where an operand comes out of another product
// (16 x 16, column l % 16, rows 4 (l / 16) + r), the indices of group q are 4q .. 4q+3 of one tile of 16 and 4q .. 4q+3 of the
// next.  bfloat16: one instruction; fp32: eight of 16 x 16 x 4, in full precision.
template <typename T> struct Operand;
template <> struct Operand<bf16> { bf16x8 v; };
template <> struct Operand<float> { float v[8]; };

template <typename T> __device__ inline Operand<T> zero_operand();
template <> __device__ inline Operand<bf16> zero_operand<bf16>() {
    Operand<bf16> o;
    const uint4 z = make_uint4(0, 0, 0, 0);
    __builtin_memcpy(&o.v, &z, 16);
    return o;
}
template <> __device__ inline Operand<float> zero_operand<float>() {
    Operand<float> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = 0.f;
    return o;
}
__device__ inline Operand<bf16> load_operand(const bf16* p) {
    Operand<bf16> o;
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    __builtin_memcpy(&o.v, &w, 16);
    return o;
}
__device__ inline Operand<float> load_operand(const float* p) {
    Operand<float> o;
    load8(p, o.v);
    return o;
}
// probabilities and their gradients as operands: bfloat16 operands round them to nearest, an error of the size of the
// rounding of the values that they multiply; sums and statistics are taken before
__device__ inline void set_operand(Operand<bf16>& o, const float (&x)[8]) {
    const uint4 w = make_uint4(cvt_pk_bf16(x[0], x[1]), cvt_pk_bf16(x[2], x[3]), cvt_pk_bf16(x[4], x[5]), cvt_pk_bf16(x[6], x[7]));
    __builtin_memcpy(&o.v, &w, 16);
}
__device__ inline void set_operand(Operand<float>& o, const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = x[i];
}
__device__ inline floatx4 product(const Operand<bf16>& a, const Operand<bf16>& b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ inline floatx4 product(const Operand<float>& a, const Operand<float>& b, floatx4 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}

// LDS rows of vectors that are read along the rows and across them: 16 bytes of padding, so that the four rows that a
// transposing read takes at once lie in different banks
template <typename T, int DP> struct TileRow { static constexpr int stride = DP + 16 / (int)sizeof(T); };

// operand with column (or row) l % 16 of 16 columns and the rows 4q .. 4q+3 and 16 + 4q .. 16 + 4q+3 of 32 LDS rows as the
// contraction indices; `tile`: first of the 32 rows at the first of the columns
template <int STRIDE>
__device__ inline Operand<bf16> across(const bf16* tile, int lane) {
    typedef short short4v __attribute__((ext_vector_type(4)));
    const int q = lane >> 4, i = lane & 15;
    const bf16* p = tile + (4 * q + (i >> 2)) * STRIDE + (i & 3) * 4;
    typedef __attribute__((address_space(3))) short4v* lds4;
    union { short4v s[2]; bf16x8 v; } u;
    u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p));
    u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + 16 * STRIDE));
    Operand<bf16> o;
    o.v = u.v;
    return o;
}
template <int STRIDE>
__device__ inline Operand<float> across(const float* tile, int lane) {
    const int q = lane >> 4, i = lane & 15;
    Operand<float> o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        o.v[j] = tile[(4 * q + j) * STRIDE + i];
        o.v[4 + j] = tile[(16 + 4 * q + j) * STRIDE + i];
    }
    return o;
}

template <int WIDTH>
__device__ inline float lanes_sum(float x) {        // over groups of WIDTH consecutive lanes
#pragma unroll
    for (int d = WIDTH / 2; d >= 1; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

}  // namespace mst
