// The products of the loss over the vocabulary on the matrix cores, and what becomes of their results before they reach memory:
//   z = h E^T            -> statistics of its rows, or the gradient dz
//   dh = dz E, dE = dz^T h
// Operands are bfloat16, or fp32 numbers split beforehand into three bfloat16 parts, of which six products are formed (the three left out are below 2^-24 of
// a term).  They go straight to LDS as they are in memory, 32 contraction indices a step; where a row of memory is one contraction index,
// ds_read_b64_tr_b16 turns four of them round on the way out.
// Rows past the end of an operand are read as its last row; what meets them is 0 on the other side, or not stored.
#include <type_traits>

#include "split_bf16.h"
#include "vocab_loss.h"

namespace mst {
namespace {

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4* lds_shortx4;

constexpr float LOG2E = 1.44269504f;

// parts of a term, the small ones first
__device__ __constant__ const int8_t PART_A[6] = {0, 2, 1, 0, 1, 0}, PART_B[6] = {2, 0, 1, 1, 0, 0};

// LDS position of unit u (eight k) of row m of an operand along: the sixteen rows of a read cover all banks
__device__ __forceinline__ uint32_t along_unit(int m, int u) {
    const int rho = (m & ~15) | ((m & 3) << 2) | ((m >> 2) & 3);
    return (uint32_t)(rho * 64 + (((u ^ (rho >> 2)) & 3) << 4));
}
// The 32-byte units (16 columns) of row k of an operand across are kept at unit ^ swizzle(k): so do the eight rows of half a wavefront
__device__ __forceinline__ int across_swizzle(int k) { return (k & 3) | ((k >> 1) & 4); }

// ---- 128 x 128 tiles, four wavefronts of 64 x 64
constexpr int SM = 128, S_OP = SM * 64;

enum Epilogue { STATS, LOGIT_GRAD, SUMS, OUT };
template <Epilogue E> struct EpilogueArgs;
template <> struct EpilogueArgs<STATS> { using type = VocabStats; };
template <> struct EpilogueArgs<LOGIT_GRAD> { using type = VocabLogitGrad; };
template <> struct EpilogueArgs<SUMS> { using type = VocabSums; };
template <> struct EpilogueArgs<OUT> { using type = VocabOut; };

// Results: acc[i][j][v] is row m0 + 16 i + lane % 16, column n0 + 16 j + 4 (lane / 16) + v of C.
// Statistics of the rows over the columns below n (n: of the piece)
template <int I, int J>
__device__ inline void finish(const VocabStats& e, const VocabProduct& p, floatx4 (&acc)[I][J], int m0, int n0, int, int lane, int) {
    const int g = lane >> 4;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                if (n0 + 16 * j + 4 * g + v >= p.n) acc[i][j][v] = -INFINITY;
                top = fmaxf(top, acc[i][j][v]);
            }
        top = apart<32>(apart<16>(top, [](float a, float b) { return fmaxf(a, b); }), [](float a, float b) { return fmaxf(a, b); });
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) sum += exp2_fast((acc[i][j][v] - base) * LOG2E);
        sum = apart<32>(apart<16>(sum, [](float a, float b) { return a + b; }), [](float a, float b) { return a + b; });
        if (g == 0 && n0 < p.n) e.stats[(int64_t)(e.first + n0 / STAT_COLUMNS) * e.row_stride + m0 + 16 * i + lane] = make_float2(top, sum);
    }
}
template <int I, int J>
__device__ inline void finish(const VocabLogitGrad& e, const VocabProduct& p, floatx4 (&acc)[I][J], int m0, int n0, int, int lane, int) {
    const int g = lane >> 4;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int m = m0 + 16 * i + (lane & 15);
        const float lse = e.lse[m], d = e.d[m], at_label = e.at_label[m];
        const int label = e.label[m] - e.v0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int n = n0 + 16 * j + 4 * g;
            float x[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                x[v] = n + v < p.n ? d * exp2_fast((acc[i][j][v] - lse) * LOG2E) : 0.f;
                if (n + v == label) x[v] = at_label;
            }
            uint16_t* const to = e.ds + (int64_t)m * e.ld + n;
            for (int q = 0; q < p.planes; ++q) {
                const uint32_t a = pack2(x[0], x[1]), b = pack2(x[2], x[3]);
                *reinterpret_cast<uint2*>(to + q * e.plane) = make_uint2(a, b);
                x[0] -= __uint_as_float(a << 16);
                x[1] -= __uint_as_float(a & 0xFFFF0000u);
                x[2] -= __uint_as_float(b << 16);
                x[3] -= __uint_as_float(b & 0xFFFF0000u);
            }
        }
    }
}
template <int I, int J>
__device__ inline void finish(const VocabSums& e, const VocabProduct& p, floatx4 (&acc)[I][J], int m0, int n0, int split, int lane, int m_rows) {
    float* const sums = e.sums + split * e.stride;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int m = m0 + 16 * i + (lane & 15);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int n = n0 + 16 * j + 4 * (lane >> 4);
            if (m >= m_rows || n >= p.n) continue;
            float4* const to = reinterpret_cast<float4*>(sums + (int64_t)m * e.ld + n);
            float4 x = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
            if (e.add) {
                const float4 o = *to;
                x = make_float4(x.x + o.x, x.y + o.y, x.z + o.z, x.w + o.w);
            }
            *to = x;
        }
    }
}
template <int I, int J>
__device__ inline void finish(const VocabOut& e, const VocabProduct& p, floatx4 (&acc)[I][J], int m0, int n0, int, int lane, int m_rows) {
    const float u = *e.unit;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int m = m0 + 16 * i + (lane & 15);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int n = n0 + 16 * j + 4 * (lane >> 4);
            if (m >= m_rows || n >= p.n) continue;                  // (n a multiple of four, as p.n is)
            const floatx4 x = acc[i][j] * u;
            if (e.f32) store4(static_cast<float*>(e.out) + (int64_t)m * e.ld + n, x[0], x[1], x[2], x[3]);
            else store4(static_cast<bf16*>(e.out) + (int64_t)m * e.ld + n, x[0], x[1], x[2], x[3]);
        }
    }
}

template <bool A_ALONG, bool B_ALONG, Epilogue E>
__global__ __launch_bounds__(256) void k_vocab_small(const VocabProduct p, const typename EpilogueArgs<E>::type e) {
    __shared__ __attribute__((aligned(16))) char lds[2 * S_OP];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m_rows = p.m_count ? *p.m_count : p.m, k_all = ((p.k_count ? *p.k_count : p.k) + VK - 1) / VK;
    const int gm = (int)((m_rows + SM - 1) / SM), gn = (p.n + SM - 1) / SM, ntiles = gm * gn;
    const int split = blockIdx.x % p.splits, tile = blockIdx.x / p.splits;
    if (tile >= ntiles) return;
    const int m0 = tile % gm * SM, n0 = tile / gm * SM;
    const int per = (k_all + p.splits - 1) / p.splits, kb = min(split * per, k_all), ke = min(kb + per, k_all);
    const uint32_t lds0 = lds_address(lds);
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;

    auto load = [&](const VocabOperand& o, auto along, int part, int t, int first, uint32_t to) __attribute__((always_inline)) {
        const uint16_t* const from = o.p + part * o.plane;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int piece = 2 * wave + j;                         // 1 KB
            const uint16_t* at;
            if constexpr (decltype(along)::value) {
                const int rho = lane >> 2, row = first + 16 * piece + (((rho & 3) << 2) | (rho >> 2)), u = ((lane & 3) ^ (rho >> 2)) & 3;
                at = from + (int64_t)min(row, o.rows - 1) * o.ld + t * VK + 8 * u;
            } else {
                const int k = 4 * piece + (lane >> 4), col = 16 * (((lane & 15) >> 1) ^ across_swizzle(k)) + 8 * (lane & 1);
                at = from + (int64_t)min(t * VK + k, o.rows - 1) * o.ld + min((int64_t)first + col, o.ld - 8);
            }
            gather_to_lds(at, to + 1024u * piece);
        }
    };
    auto read = [&](auto along, uint32_t op, int first) __attribute__((always_inline)) {
        if constexpr (decltype(along)::value) {
            return *reinterpret_cast<const bf16x8*>(lds + op + along_unit(first + (lane & 15), lane >> 4));
        } else {
            const int g = lane >> 4, x = (lane >> 2) & 3, k = 8 * g + x;
            const uint32_t at = lds0 + op + (uint32_t)(k * SM * 2 + (((first >> 4) ^ across_swizzle(k)) << 5) + (lane & 3) * 8);
            // (four rows further on: the same swizzle)
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(uintptr_t)at);
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(uintptr_t)(at + 4 * SM * 2));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };

    floatx4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int term = p.planes == 1 ? 5 : 0; term < 6; ++term)
        for (int t = kb; t < ke; ++t) {
            __syncthreads();
            load(p.a, std::bool_constant<A_ALONG>{}, PART_A[term], t, m0, lds0);
            load(p.b, std::bool_constant<B_ALONG>{}, PART_B[term], t, n0, lds0 + S_OP);
            wait_loads<0>();
            __syncthreads();
            bf16x8 a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = read(std::bool_constant<A_ALONG>{}, 0, wm + 16 * i);
                b[i] = read(std::bool_constant<B_ALONG>{}, S_OP, wn + 16 * i);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
        }
    finish(e, p, acc, m0 + wm, n0 + wn, split, lane, m_rows);
}

template <bool A_ALONG, bool B_ALONG, Epilogue E>
int launch(const VocabProduct& p, const typename EpilogueArgs<E>::type& e, hipStream_t s) {
    const int64_t blocks = cdiv(p.m, SM) * cdiv(p.n, SM) * p.splits;
    k_vocab_small<A_ALONG, B_ALONG, E><<<(unsigned)blocks, 256, 0, s>>>(p, e);
    MST_LAUNCH_CHECK();
    return MST_OK;
}

}  // namespace

int vocab_stats(const VocabProduct& p, const VocabStats& e, hipStream_t s) { return launch<true, true, STATS>(p, e, s); }
int vocab_logit_grad(const VocabProduct& p, const VocabLogitGrad& e, hipStream_t s) { return launch<true, true, LOGIT_GRAD>(p, e, s); }
int vocab_sums(const VocabProduct& p, const VocabSums& e, hipStream_t s) { return launch<true, false, SUMS>(p, e, s); }
int vocab_out(const VocabProduct& p, const VocabOut& e, hipStream_t s) { return launch<false, false, OUT>(p, e, s); }

}  // namespace mst
