// Heads of queries, keys and values as the attention half of a block reads and writes them: strided views of vectors of
// head_dim contiguous components, their checks on the host, 16-byte loads and the operands of the matrix instructions.
#pragma once

#include "common.h"
#include "split_bf16.h"

namespace mst {

constexpr int HEAD_DIM_MAX = 128;        // of the attention; head_dim is a multiple of 8
constexpr int SELECT_MAX = 64, SELECT_BITS = 6;      // blocks a query may select; a pair is query << 6 | place in its row
constexpr int KEY_BLOCKS_MAX = 2048;     // blocks of a sequence: their bit words for 256 queries are 64 KB of LDS
constexpr int64_t HEADS_MAX = 1 << 16;
constexpr int LDS_BYTES = 160 * 1024;     // of a CU

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

// {bf16(a), bf16(b)}, to nearest even: the instruction of cvt_pk_bf16 from the compiler itself, which knows that a number straight out
// of an exponential has to be waited for (written as asm it has been read too early)
__device__ inline uint32_t pack2(float a, float b) {
    typedef float float2v __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = __builtin_convertvector((float2v{a, b}), bf16x2);
    uint32_t r;
    __builtin_memcpy(&r, &v, 4);
    return r;
}

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
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
}
__device__ inline void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ inline void store4(bf16* p, float a, float b, float c, float d) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2(a, b), pack2(c, d));
}

// ---- operands of a 32 x 32 x 16 product.  Lane l holds row (or column) l % 32 and the eight contraction indices of half l / 32.
// Which eight is free as long as both operands agree.  Rows of a result: 8 (r / 4) + 4 (l / 32) + r % 4 in register r, column
// l % 32; where a result is the next operand, half h of sixteen indices has 4h .. 4h+3 and 8 + 4h .. 8 + 4h+3, which are its registers
// 8i .. 8i+7 in order.  bfloat16: one instruction; fp32: eight of 32 x 32 x 2, in full precision.
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
    const uint4 w = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
    __builtin_memcpy(&o.v, &w, 16);
}
__device__ inline void set_operand(Operand<float>& o, const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = x[i];
}
__device__ inline void numbers(const Operand<bf16>& o, float (&x)[8]) {
    uint4 w;
    __builtin_memcpy(&w, &o.v, 16);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
}
__device__ inline void numbers(const Operand<float>& o, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = o.v[e];
}
// what the rounding to `o` left: x - o, rounded in turn
__device__ inline void set_operand_rest(Operand<bf16>& rest, const Operand<bf16>& o, const float (&x)[8]) {
    uint4 w;
    __builtin_memcpy(&w, &o.v, 16);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[2 * i] = x[2 * i] - __uint_as_float(u[i] << 16), y[2 * i + 1] = x[2 * i + 1] - __uint_as_float(u[i] & 0xFFFF0000u);
    set_operand(rest, y);
}
__device__ inline void set_operand_rest(Operand<float>&, const Operand<float>&, const float (&)[8]) {}
__device__ inline floatx16 product32(const Operand<bf16>& a, const Operand<bf16>& b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ inline floatx16 product32(const Operand<float>& a, const Operand<float>& b, floatx16 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}
// components from `d` on are there?  fp32 products take eight instructions, each twice the time of bfloat16's one: they are left out where
// head_dim ends before the padded width does (80 components: 5 of 8 and 3 of 4; the scores of dQ's walk still go through all).  bfloat16 ones are
// not worth the branch: with it forward and gradients of 4096 queries take 504 us against 478 at 80 components, 481 against 442 at 96; of 8192 at 40
// 560 against 550, at 64 563 against 540, and at 32 alone 484 against 522.
template <typename T>
__device__ inline bool worth(int d, int D) { return sizeof(T) == 2 || d == 0 || d < D; }
__device__ inline floatx16 zero16() {
    floatx16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}
// ---- LDS tiles of vectors that are read along the rows and across them.  A row is CH chunks of 16 bytes; chunk c of row r is
// kept at place c ^ mix(r): eight consecutive rows then have a chunk in eight different places (a read along the rows takes
// 16 bytes from each), and four consecutive rows, from a multiple of four on, have four neighbouring chunks in different ones (a
// transposing read of 32 columns).  Lanes that load straight to LDS write a row's places in order and pick the chunks.
template <typename T, int DP>
struct Rows {
    static constexpr int CH = DP * (int)sizeof(T) / 16, BYTES = CH * 16, PER_KB = 64 / CH;      // rows of one load of a wavefront
    __device__ static int mix(int r) { return CH == 8 ? ((r & 2) << 1) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3); }
    __device__ static int at(int r, int c) { return r * BYTES + ((c ^ mix(r)) << 4); }
};
template <int DP>
__device__ inline Operand<bf16> along(const char* tile, int r, int d) {            // components d .. d+7 of row r
    Operand<bf16> o;
    o.v = *reinterpret_cast<const bf16x8*>(tile + Rows<bf16, DP>::at(r, d >> 3));
    return o;
}
template <int DP>
__device__ inline Operand<float> along_f32(const char* tile, int r, int d) {
    Operand<float> o;
    const float4 a = *reinterpret_cast<const float4*>(tile + Rows<float, DP>::at(r, d >> 2)), b = *reinterpret_cast<const float4*>(tile + Rows<float, DP>::at(r, (d >> 2) + 1));
    o.v[0] = a.x; o.v[1] = a.y; o.v[2] = a.z; o.v[3] = a.w;
    o.v[4] = b.x; o.v[5] = b.y; o.v[6] = b.z; o.v[7] = b.w;
    return o;
}
// column d0 + l % 32 of the rows r0 .. r0+15 as contraction indices, in the order of a result; r0 a multiple of 16
template <int DP>
__device__ inline Operand<bf16> across(const char* tile, int r0, int d0, int lane) {
    typedef short short4v __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4v* lds4;
    const int i = lane & 15, r = r0 + 4 * (lane >> 5) + (i >> 2), d = d0 + ((lane >> 4) & 1) * 16 + (i & 3) * 4;
    union { short4v s[2]; bf16x8 v; } u;
    u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(tile + Rows<bf16, DP>::at(r, d >> 3) + (d & 7) * 2));
    u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(tile + Rows<bf16, DP>::at(r + 8, d >> 3) + (d & 7) * 2));
    Operand<bf16> o;
    o.v = u.v;
    return o;
}
template <int DP>
__device__ inline Operand<float> across_f32(const char* tile, int r0, int d0, int lane) {
    const int d = d0 + (lane & 31), r = r0 + 4 * (lane >> 5);
    Operand<float> o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        o.v[j] = *reinterpret_cast<const float*>(tile + Rows<float, DP>::at(r + j, d >> 2) + (d & 3) * 4);
        o.v[4 + j] = *reinterpret_cast<const float*>(tile + Rows<float, DP>::at(r + 8 + j, d >> 2) + (d & 3) * 4);
    }
    return o;
}
template <typename T, int DP>
__device__ inline Operand<T> along_row(const char* tile, int r, int d) {
    if constexpr (sizeof(T) == 2) return along<DP>(tile, r, d);
    else return along_f32<DP>(tile, r, d);
}
template <typename T, int DP>
__device__ inline Operand<T> across_rows(const char* tile, int r0, int d0, int lane) {
    if constexpr (sizeof(T) == 2) return across<DP>(tile, r0, d0, lane);
    else return across_f32<DP>(tile, r0, d0, lane);
}
// 16 bytes per lane from its own address to LDS, lane l to lds + 16 l
__device__ __forceinline__ void gather_to_lds(const void* from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)(const char*)p);
}
template <typename T> __device__ inline Operand<T> negated(Operand<T> o) {
    uint32_t w[sizeof(o.v) / 4];
    __builtin_memcpy(w, &o.v, sizeof(o.v));
#pragma unroll
    for (auto& x : w) x ^= sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
    __builtin_memcpy(&o.v, w, sizeof(o.v));
    return o;
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }    // results below 2^-126 are 0

// Rows of 16 lanes: both numbers of lanes 16 (or 32) apart, the even row's (the lower half's) first, in either of them
struct Both { uint32_t first, second; };
template <int APART>
__device__ inline Both both_lanes(uint32_t x) {
    typedef unsigned uint2v __attribute__((ext_vector_type(2)));
    uint2v r;
    if constexpr (APART == 16) r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    else r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return {r[0], r[1]};
}
template <int APART, typename V, typename F>
__device__ inline V apart(V x, F&& f) {
    const Both b = both_lanes<APART>(__builtin_bit_cast(uint32_t, x));
    return f(__builtin_bit_cast(V, b.first), __builtin_bit_cast(V, b.second));
}
// f(x, the same of another lane) over groups of WIDTH consecutive lanes, WIDTH up to 64; every lane gets the result.  Within 16 lanes the
// other lane's number comes with the instruction (pairs, pairs of pairs, mirrored eights, mirrored rows).
template <int CONTROL>
__device__ inline float other_lane(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CONTROL, 0xF, 0xF, true)); }
template <int CONTROL>
__device__ inline int other_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, CONTROL, 0xF, 0xF, true); }
template <int WIDTH, typename V, typename F>
__device__ inline V over_lanes(V x, F&& f) {
    if (WIDTH >= 2) x = f(x, other_lane<0xB1>(x));
    if (WIDTH >= 4) x = f(x, other_lane<0x4E>(x));
    if (WIDTH >= 8) x = f(x, other_lane<0x141>(x));
    if (WIDTH >= 16) x = f(x, other_lane<0x140>(x));
    if (WIDTH >= 32) x = apart<16>(x, f);
    if (WIDTH >= 64) x = apart<32>(x, f);
    return x;
}
// in rows of 16 lanes: the sum of x over this row and the odd one behind it where the row is even, else that of y over the one before and this
__device__ inline float sixteen_apart_sum(float x, float y) {
    typedef unsigned uint2v __attribute__((ext_vector_type(2)));
    const uint2v r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int WIDTH>
__device__ inline float lanes_sum(float x) { return over_lanes<WIDTH>(x, [](float a, float b) { return a + b; }); }
template <int WIDTH>
__device__ inline float lanes_max(float x) { return over_lanes<WIDTH>(x, [](float a, float b) { return fmaxf(a, b); }); }
template <int WIDTH>
__device__ inline int lanes_max(int x) { return over_lanes<WIDTH>(x, [](int a, int b) { return max(a, b); }); }

}  // namespace mst
