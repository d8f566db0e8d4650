// Which blocks of keys a query reads: 8-bit summaries of the blocks, scores in whole numbers, the best of them, and the plan
// that turns a selection into lists of queries.
//
// Keys and queries are scaled by powers of two and rounded to 8 bits, summed as whole numbers and rounded to 8 bits again; a
// score is a sum of at most 128 products below 2^14, exact in 32 bits, times the block's power of two.  Nothing here depends on
// the order of a sum, so every kernel below may split its work as it likes.
#include "block_attention.h"

namespace mst {
namespace {

constexpr int E_MAX = 100;               // exponents of the largest component are taken into -E_MAX .. E_MAX

__device__ inline float power_of_two(int e) { return __int_as_float((e + 127) << 23); }      // -126 <= e <= 127
// floor(log2 x) of fp32 x >= 0, below -126 for zero and subnormal numbers
__device__ inline int exponent(float x) { return (int)(__float_as_uint(x) >> 23) - 127; }
__device__ inline int unit_exponent(float top) { return min(max(exponent(top), -E_MAX), E_MAX); }
__device__ inline float finite_or_0(float x) { return fabsf(x) <= 3.402823466e38f ? x : 0.f; }
__device__ inline int round8(float x) { return (int)fminf(fmaxf(rintf(x), -127.f), 127.f); }
// shift that brings whole numbers up to `top` into 8 bits
__device__ inline int sum_shift(int top) { return top > 0 ? max(31 - __clz(top) - 6, 0) : 0; }

// ---- summaries: a workgroup per block of keys.  A thread holds one unit of eight components of every (256 / units)-th key in
// registers, so keys are read once.
constexpr int SUM_THREADS = 256;
template <typename T>
__global__ __launch_bounds__(SUM_THREADS) void k_key_summary(AttentionArgs a, Heads<const T> k, int8_t* __restrict__ sums, float* __restrict__ scales,
                                                             int new_tokens) {
    __shared__ int part[HEAD_DIM_MAX];
    __shared__ float top4[4];
    __shared__ int peak4[4];
    const int bg = blockIdx.y, b = bg / a.G, g = bg % a.G, len = a.length(b);
    const int first = new_tokens >= len ? 0 : (len - new_tokens) / a.BK;
    const int j = first + blockIdx.x;
    if (j >= len / a.BK) return;
    const int units = a.D / 8, per = SUM_THREADS / units;      // 16 .. 256 keys at a time
    const int u = threadIdx.x % units, k0 = threadIdx.x / units;
    const bool mine = k0 < per;
    const T* base = k.at(b, (int64_t)j * a.BK, g) + u * 8;
    for (int i = threadIdx.x; i < a.D; i += SUM_THREADS) part[i] = 0;
    float top = 0.f;
    if (mine)
        for (int r = k0; r < a.BK; r += per) {
            float x[8];
            load8(base + r * k.st, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(finite_or_0(x[e])));
        }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((threadIdx.x & 63) == 0) top4[threadIdx.x >> 6] = top;
    __syncthreads();
    const int E = unit_exponent(fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])));
    const float unit = power_of_two(6 - E);
    if (mine) {
        int s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int r = k0; r < a.BK; r += per) {
            float x[8];
            load8(base + r * k.st, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += round8(finite_or_0(x[e]) * unit);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) atomicAdd(&part[u * 8 + e], s[e]);
    }
    __syncthreads();
    const int v = (int)threadIdx.x < a.D ? part[threadIdx.x] : 0;
    int peak = abs(v);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) peak = max(peak, __shfl_xor(peak, d));
    if ((threadIdx.x & 63) == 0) peak4[threadIdx.x >> 6] = peak;
    __syncthreads();
    const int shift = sum_shift(max(max(peak4[0], peak4[1]), max(peak4[2], peak4[3])));
    const int64_t at = (int64_t)bg * a.nb + j;
    if ((int)threadIdx.x < a.D) sums[at * a.D + threadIdx.x] = (int8_t)round8((float)v * power_of_two(-shift));
    if (threadIdx.x == 0) scales[at] = power_of_two(E - 6 + shift);
}

// ---- a query in 8 bits: the sixteen lanes of a query hold eight components each (lane c: 8c ..), over its R heads
template <typename T>
__device__ inline uint2 query8(const AttentionArgs& a, const Heads<const T>& q, int b, int t, int g, int c, bool there) {
    const bool mine = there && c * 8 < a.D;
    float top = 0.f;
    if (mine)
        for (int h = 0; h < a.R; ++h) {
            float x[8];
            load8(q.at(b, t, g * a.R + h) + c * 8, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(finite_or_0(x[e])));
        }
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float unit = power_of_two(6 - unit_exponent(top));
    int s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (mine)
        for (int h = 0; h < a.R; ++h) {
            float x[8];
            load8(q.at(b, t, g * a.R + h) + c * 8, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += round8(finite_or_0(x[e]) * unit);
        }
    int peak = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) peak = max(peak, abs(s[e]));
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) peak = max(peak, __shfl_xor(peak, d));
    const float back = power_of_two(-sum_shift(peak));
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e >> 2] |= (uint32_t)(round8((float)s[e] * back) & 255) << (8 * (e & 3));
    return make_uint2(w[0], w[1]);
}

// scores as unsigned numbers of the same order; 0 (below every score) for no candidate
__device__ inline uint32_t ordered(float x) {
    x += 0.f;                                                  // -0 and +0 are one score
    const uint32_t u = __float_as_uint(x);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// ---- selection, a wavefront per 64 queries.  16 blocks at a time the scores come from the 8-bit matrix instructions, go through
// LDS and to the query's own lane, which keeps the KK highest in order: one median a place.  With the lowest of them known a second
// walk over the same scores takes the blocks above it and, on a tie, the first that are due, in ascending order.
typedef int intx4 __attribute__((ext_vector_type(4)));
template <typename T, int KK>
__global__ __launch_bounds__(64) void k_block_select(AttentionArgs a, Heads<const T> q, const int8_t* __restrict__ sums,
                                                     const float* __restrict__ scales, int* __restrict__ blocks) {
    __shared__ __align__(16) uint2 q8[64][17];                 // a query's 128 components; 8 bytes of padding
    __shared__ uint32_t score[16][65];
    const int bg = blockIdx.y, b = bg / a.G, g = bg % a.G, len = a.length(b);
    const int lane = threadIdx.x, i = lane & 15, quad = lane >> 4;
    const int t0 = blockIdx.x * 64;
    for (int r = quad; r < 64; r += 4) q8[r][i] = query8(a, q, b, t0 + r, g, i, t0 + r < a.Tq && len - a.Tq + t0 + r >= 0);
    __syncthreads();
    intx4 qb[4][2];                                            // column = query, 16 components of every 64 to a lane
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const uint2 lo = q8[n * 16 + i][c * 8 + quad * 2], hi = q8[n * 16 + i][c * 8 + quad * 2 + 1];
            qb[n][c] = intx4{(int)lo.x, (int)lo.y, (int)hi.x, (int)hi.y};
        }
    const int t = t0 + lane, p = len - a.Tq + t;
    const bool there = t < a.Tq && p >= 0;
    const int mine = there ? p / a.BK : 0;                     // candidates: the blocks before it
    const int last_t = min(t0 + 63, a.Tq - 1), last_p = len - a.Tq + last_t;
    const int most = last_p >= 0 ? last_p / a.BK : 0;
    const int8_t* srow = sums + (int64_t)bg * a.nb * a.D;
    const float* scl = scales + (int64_t)bg * a.nb;
    const int wanted = a.NS - 1;
    auto scores = [&](int j0) {
        intx4 ab[2] = {intx4{0, 0, 0, 0}, intx4{0, 0, 0, 0}};  // row = block
        const int j = j0 + i;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int d = c * 64 + quad * 16;
            if (j < most && d < a.D) {                         // (rows are whole eights of bytes, at eights)
                const uint2* s = reinterpret_cast<const uint2*>(srow + (int64_t)j * a.D + d);
                const uint2 lo = s[0], hi = d + 8 < a.D ? s[1] : make_uint2(0, 0);
                ab[c] = intx4{(int)lo.x, (int)lo.y, (int)hi.x, (int)hi.y};
            }
        }
        float unit[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) unit[r] = j0 + 4 * quad + r < most ? scl[j0 + 4 * quad + r] : 0.f;
        __syncthreads();                                       // (one wavefront: the reads of the scores before these)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            intx4 c = {0, 0, 0, 0};
            c = __builtin_amdgcn_mfma_i32_16x16x64_i8(ab[0], qb[n][0], c, 0, 0, 0);
            if (a.D > 64) c = __builtin_amdgcn_mfma_i32_16x16x64_i8(ab[1], qb[n][1], c, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) score[4 * quad + r][n * 16 + i] = ordered((float)c[r] * unit[r]);
        }
        __syncthreads();
    };
    uint32_t best[KK];                                         // descending; the places past `wanted` are taken from the start
#pragma unroll
    for (int e = 0; e < KK; ++e) best[e] = e < KK - wanted ? 0xFFFFFFFFu : 0u;
    if (wanted > 0)
        for (int j0 = 0; j0 < most; j0 += 16) {
            scores(j0);
#pragma unroll 4
            for (int r = 0; r < 16; ++r) {
                const uint32_t v = j0 + r < mine ? score[r][lane] : 0u;
                if (__any(v > best[KK - 1])) {
#pragma unroll
                    for (int e = KK - 1; e > 0; --e) {         // median of v and two neighbours: v sinks to its place
                        const uint32_t hi = best[e - 1], lo = best[e];
                        best[e] = max(min(v, hi), lo);
                    }
                    best[0] = max(v, best[0]);
                }
            }
        }
    const uint32_t least = best[KK - 1];
    int due = 0;                                               // how many equal to the lowest one are taken
#pragma unroll
    for (int e = 0; e < KK; ++e) due += (e >= KK - wanted && best[e] == least) ? 1 : 0;
    int* out = blocks + ((int64_t)bg * a.Tq + t) * a.NS;
    int n = 0;
    if (wanted > 0)
        for (int j0 = 0; j0 < most; j0 += 16) {
            scores(j0);
            for (int r = 0; r < 16; ++r) {
                const uint32_t v = score[r][lane];
                if (j0 + r < mine && (v > least || (v == least && due > 0))) {
                    if (v == least) --due;
                    out[n++] = j0 + r;
                }
            }
        }
    if (t < a.Tq) {
        if (there) out[n++] = mine;
        for (; n < a.NS; ++n) out[n] = -1;
    }
}

// ---- selection for few queries: a workgroup per query and key head.  Scores in LDS; the lowest that is taken is found bit by
// bit, the workgroup counting the scores at or above a trial value.
constexpr int FEW_THREADS = 256;
template <typename T>
__global__ __launch_bounds__(FEW_THREADS) void k_block_select_few(AttentionArgs a, Heads<const T> q, const int8_t* __restrict__ sums,
                                                                  const float* __restrict__ scales, int* __restrict__ blocks) {
    __shared__ __align__(16) uint2 q8[16];
    __shared__ uint32_t score[KEY_BLOCKS_MAX];
    __shared__ int count[2][4];
    __shared__ int before[FEW_THREADS];
    const int bg = blockIdx.y, b = bg / a.G, g = bg % a.G, len = a.length(b), t = blockIdx.x;
    const int p = len - a.Tq + t, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int* out = blocks + ((int64_t)bg * a.Tq + t) * a.NS;
    if (p < 0) {
        for (int n = threadIdx.x; n < a.NS; n += FEW_THREADS) out[n] = -1;
        return;
    }
    const int mine = p / a.BK, wanted = min(a.NS - 1, mine);
    if (wave == 0) {
        const uint2 w = query8(a, q, b, t, g, lane & 15, true);
        if (lane < 16) q8[lane] = w;
    }
    __syncthreads();
    const int8_t* srow = sums + (int64_t)bg * a.nb * a.D;
    const float* scl = scales + (int64_t)bg * a.nb;
    for (int j = threadIdx.x; j < mine; j += FEW_THREADS) {
        const uint2* s = reinterpret_cast<const uint2*>(srow + (int64_t)j * a.D);
        int dot = 0;
        for (int u = 0; u < a.D / 8; ++u) {
            const uint2 w = s[u], x = q8[u];
            dot = __builtin_amdgcn_sdot4((int)w.x, (int)x.x, dot, false);
            dot = __builtin_amdgcn_sdot4((int)w.y, (int)x.y, dot, false);
        }
        score[j] = ordered((float)dot * scl[j]);
    }
    __syncthreads();
    // the highest value with at least `wanted` scores at or above it
    uint32_t least = 0;
    if (wanted > 0 && wanted < mine)
        for (int bit = 31, turn = 0; bit >= 0; --bit, turn ^= 1) {
            const uint32_t trial = least | (1u << bit);
            int c = 0;
            for (int j = threadIdx.x; j < mine; j += FEW_THREADS) c += score[j] >= trial;
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) c += __shfl_xor(c, d);
            if (lane == 0) count[turn][wave] = c;
            __syncthreads();
            const int all = count[turn][0] + count[turn][1] + count[turn][2] + count[turn][3];
            if (all >= wanted) least = trial;
            if (all == wanted) break;
        }
    // every thread takes a stretch of blocks: its number above and equal, then its places
    const int each = (mine + FEW_THREADS - 1) / FEW_THREADS, j0 = threadIdx.x * each, j1 = min(j0 + each, mine);
    int above = 0, equal = 0;
    if (wanted > 0)
        for (int j = j0; j < j1; ++j) {
            above += score[j] > least;
            equal += score[j] == least;
        }
    before[threadIdx.x] = above << 16 | equal;                 // (up to 2048 of either)
    __syncthreads();
    int a0 = 0, e0 = 0, total_above = 0;
    for (int i = 0; i < FEW_THREADS; ++i) {
        const int w = before[i];
        if (i < (int)threadIdx.x) a0 += w >> 16, e0 += w & 0xFFFF;
        total_above += w >> 16;
    }
    const int ties = wanted - total_above;                     // of the equal ones, the first so many
    if (wanted > 0)
        for (int j = j0; j < j1; ++j) {
            const uint32_t v = score[j];
            if (v > least || (v == least && e0 < ties)) out[a0 + min(e0, ties)] = j;
            if (v > least) ++a0;
            else if (v == least) ++e0;
        }
    if (threadIdx.x == 0) out[wanted] = mine;
    for (int n = wanted + 1 + threadIdx.x; n < a.NS; n += FEW_THREADS) out[n] = -1;
}

// ---- plan.  A tile of 256 queries marks its queries in one bit word of 256 a block: a query has a block once at most, so the number
// of bits below its own is its place among the tile's.  Counts per tile, their sums over the tiles, then every pair to its place.
__device__ inline void mark_tile(const AttentionArgs& a, const int* __restrict__ blocks, int bg, int t, int len, uint32_t* bits, int* rows_out) {
    for (int i = threadIdx.x; i < a.nb * 8; i += PLAN_TILE) bits[i] = 0;
    __syncthreads();
    if (t < a.Tq) {
        const int p = len - a.Tq + t, own = p >= 0 ? p / a.BK : -1;
        const int* row = blocks + ((int64_t)bg * a.Tq + t) * a.NS;
        int* out = rows_out + ((int64_t)bg * a.Tq + t) * a.NS;
        int last = -1, n = 0;
        for (int s = 0; s < a.NS; ++s) {
            const int j = row[s];
            if (j > last && j <= own) {
                out[n++] = j;
                atomicOr(&bits[j * 8 + (threadIdx.x >> 5)], 1u << (threadIdx.x & 31));
                last = j;
            }
        }
        for (; n < a.NS; ++n) out[n] = a.nb;
    }
    __syncthreads();
}

__global__ __launch_bounds__(PLAN_TILE) void k_plan_count(AttentionArgs a, const int* __restrict__ blocks, Plan plan) {
    extern __shared__ uint32_t bits[];
    const int bg = blockIdx.y, t = blockIdx.x * PLAN_TILE + threadIdx.x;
    mark_tile(a, blocks, bg, t, a.length(bg / a.G), bits, plan.rows);
    int* row = plan.tile + ((int64_t)bg * plan.tiles + blockIdx.x) * a.nb;
    for (int j = threadIdx.x; j < a.nb; j += PLAN_TILE) {
        int c = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) c += __popc(bits[j * 8 + w]);
        row[j] = c;
    }
}

// exclusive sums of two numbers over the threads of a workgroup of 1024
__device__ inline int2 exclusive(int2 v, int2* total) {
    __shared__ int2 wave_sum[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int2 x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int px = __shfl_up(x.x, d), py = __shfl_up(x.y, d);
        if (lane >= d) x.x += px, x.y += py;
    }
    if (lane == 63) wave_sum[wave] = x;
    __syncthreads();
    int2 before = make_int2(0, 0), all = make_int2(0, 0);
    for (int w = 0; w < 16; ++w) {
        const int2 s = wave_sum[w];
        if (w < wave) before.x += s.x, before.y += s.y;
        all.x += s.x, all.y += s.y;
    }
    __syncthreads();
    *total = all;
    return make_int2(before.x + x.x - v.x, before.y + x.y - v.y);
}

__global__ __launch_bounds__(1024) void k_plan_sums(AttentionArgs a, Plan plan) {
    const int bg = blockIdx.x;
    int* tile = plan.tile + (int64_t)bg * plan.tiles * a.nb;
    int* start = plan.start + (int64_t)bg * (a.nb + 1);
    int* item_start = plan.item_start + (int64_t)bg * (a.nb + 1);
    int2* items = plan.items + (int64_t)bg * plan.max_items;
    int2 done = make_int2(0, 0);
    for (int j0 = 0; j0 < a.nb; j0 += 1024) {
        const int j = j0 + threadIdx.x;
        int n = 0;
        if (j < a.nb)
            for (int i = 0; i < plan.tiles; ++i) {
                const int c = tile[(int64_t)i * a.nb + j];
                tile[(int64_t)i * a.nb + j] = n;
                n += c;
            }
        const int parts = (n + plan.item_pairs - 1) / plan.item_pairs;
        int2 all;
        const int2 at = exclusive(make_int2(n, parts), &all);
        if (j < a.nb) {
            start[j] = done.x + at.x;
            item_start[j] = done.y + at.y;
            for (int i = 0; i < parts; ++i) items[done.y + at.y + i] = make_int2(j, done.x + at.x + i * plan.item_pairs);
        }
        done.x += all.x, done.y += all.y;
    }
    if (threadIdx.x == 0) start[a.nb] = done.x, item_start[a.nb] = done.y;
}

__global__ __launch_bounds__(PLAN_TILE) void k_plan_fill(AttentionArgs a, Plan plan) {
    extern __shared__ uint32_t bits[];
    const int bg = blockIdx.y, t = blockIdx.x * PLAN_TILE + threadIdx.x;
    for (int i = threadIdx.x; i < a.nb * 8; i += PLAN_TILE) bits[i] = 0;
    __syncthreads();
    const int word = threadIdx.x >> 5;
    const int* row = plan.rows + ((int64_t)bg * a.Tq + t) * a.NS;
    if (t < a.Tq)
        for (int s = 0; s < a.NS && row[s] < a.nb; ++s) atomicOr(&bits[row[s] * 8 + word], 1u << (threadIdx.x & 31));
    __syncthreads();
    if (t >= a.Tq) return;
    const int* before = plan.tile + ((int64_t)bg * plan.tiles + blockIdx.x) * a.nb;
    const int* start = plan.start + (int64_t)bg * (a.nb + 1);
    int* list = plan.list + (int64_t)bg * a.Tq * a.NS;
    for (int s = 0; s < a.NS && row[s] < a.nb; ++s) {
        const int j = row[s];
        int at = start[j] + before[j] + __popc(bits[j * 8 + word] & ((1u << (threadIdx.x & 31)) - 1));
        for (int w = 0; w < word; ++w) at += __popc(bits[j * 8 + w]);
        list[at] = t * a.NS + s;
    }
}

// fewer queries than this: a workgroup for each
constexpr int FEW_QUERIES = 16;

}  // namespace
}  // namespace mst

extern "C" int mst_key_summary(const mst_attention_shape* s, const mst_heads* k, int8_t* sums, float* scales, int new_tokens, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    if (!sums || !scales || !aligned16(sums) || !aligned16(scales) || new_tokens < 0) return MST_ERR_ARG;
    if (int e = check_heads(k, s->batch, s->keys, s->kv_heads, s->type, false)) return e;
    const AttentionArgs a = attention_args(s);
    // blocks that a sequence's last new_tokens keys can complete
    const int64_t most = std::min<int64_t>(s->keys / s->block, (int64_t)new_tokens / s->block + 1);
    if (a.B == 0 || most == 0 || new_tokens == 0) return MST_OK;
    with_type(s->type, [&](auto t) {
        using T = decltype(t);
        k_key_summary<T><<<dim3((unsigned)most, (unsigned)(a.B * a.G)), SUM_THREADS, 0, static_cast<hipStream_t>(stream)>>>(a, heads_of<const T>(k), sums, scales, new_tokens);
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}

extern "C" int mst_block_select(const mst_attention_shape* s, const mst_heads* q, const int8_t* sums, const float* scales, int32_t* blocks, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    if (!sums || !scales || !blocks || !aligned16(sums) || !aligned16(scales) || !aligned16(blocks)) return MST_ERR_ARG;
    if (int e = check_heads(q, s->batch, s->queries, s->heads, s->type, false)) return e;
    const AttentionArgs a = attention_args(s);
    if (a.B == 0 || a.Tq == 0) return MST_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    with_type(s->type, [&](auto t) {
        using T = decltype(t);
        const Heads<const T> qh = heads_of<const T>(q);
        if (a.Tq < FEW_QUERIES) {
            k_block_select_few<T><<<dim3((unsigned)a.Tq, (unsigned)(a.B * a.G)), FEW_THREADS, 0, st>>>(a, qh, sums, scales, blocks);
            return;
        }
        const dim3 grid((unsigned)cdiv(a.Tq, 64), (unsigned)(a.B * a.G));
        const int wanted = a.NS - 1;
        if (wanted <= 4) k_block_select<T, 4><<<grid, 64, 0, st>>>(a, qh, sums, scales, blocks);
        else if (wanted <= 8) k_block_select<T, 8><<<grid, 64, 0, st>>>(a, qh, sums, scales, blocks);
        else if (wanted <= 16) k_block_select<T, 16><<<grid, 64, 0, st>>>(a, qh, sums, scales, blocks);
        else if (wanted <= 32) k_block_select<T, 32><<<grid, 64, 0, st>>>(a, qh, sums, scales, blocks);
        else k_block_select<T, 63><<<grid, 64, 0, st>>>(a, qh, sums, scales, blocks);
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}

extern "C" size_t mst_block_plan_bytes(const mst_attention_shape* s) {
    using namespace mst;
    if (check_attention(s)) return 0;
    return carve_plan(nullptr, attention_args(s)).total;
}

extern "C" int mst_block_plan(const mst_attention_shape* s, const int32_t* blocks, void* plan_dev, size_t plan_bytes, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    if (!blocks || !plan_dev || !aligned16(blocks) || !aligned16(plan_dev)) return MST_ERR_ARG;
    const AttentionArgs a = attention_args(s);
    const Plan plan = carve_plan(plan_dev, a);
    if (plan_bytes < plan.total) return MST_ERR_WORKSPACE;
    if (a.B == 0) return MST_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)plan.tiles, (unsigned)(a.B * a.G));
    const size_t lds = (size_t)std::max(a.nb, 1) * 32;          // 64 KB at most
    if (plan.tiles > 0) {
        k_plan_count<<<grid, PLAN_TILE, lds, st>>>(a, blocks, plan);
        MST_LAUNCH_CHECK();
    }
    k_plan_sums<<<(unsigned)(a.B * a.G), 1024, 0, st>>>(a, plan);
    MST_LAUNCH_CHECK();
    if (plan.tiles > 0) {
        k_plan_fill<<<grid, PLAN_TILE, lds, st>>>(a, plan);
        MST_LAUNCH_CHECK();
    }
    return MST_OK;
}
