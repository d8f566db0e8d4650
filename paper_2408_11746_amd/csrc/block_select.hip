// Which blocks of keys a query reads: 8-bit summaries of the blocks, scores in whole numbers, the best of them, the plan that keeps
// the entries of a selection that count, and the lists of a block's queries that the gradients make of a plan.
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
// Whole numbers of 8 bits: x is cut at 127 units, and a number between -2^22 and 2^22 added to ROUND has its value, rounded to
// nearest even, in the low bits.  (x is finite; what is not gives some number of 8 bits.)
constexpr float ROUND = 12582912.f;      // 1.5 2^23
__device__ inline int round8_bits(float x, float unit, float most) {       // ROUND's bits + round8(x unit); most = 127 / unit
    return __float_as_int(__builtin_fmaf(__builtin_amdgcn_fmed3f(x, -most, most), unit, ROUND));
}
constexpr int ROUND_BITS = 0x4B400000;
// shift that brings whole numbers up to `top` into 8 bits
__device__ inline int sum_shift(int top) { return top > 0 ? max(31 - __clz(top) - 6, 0) : 0; }

// ---- summaries: a workgroup per block of keys.  A thread holds one unit of eight components of every (256 / units)-th key in
// registers, so keys are read once: 19 us for 32768 keys of 8 heads of 128 (67 MB, 3.5 TB/s), 10.4 for 8192 of 20 of 64 (2 TB/s: start and reductions).
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
    constexpr int PIECES = HEAD_DIM_MAX / 16;                  // 128 keys of 128 components: eight pieces a thread
    float x[PIECES][8], top = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int r = k0 + i * per;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
        if (mine && r < a.BK) load8(base + r * k.st, x[i]);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
        if (i * per < a.BK)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[i][e]));
    top = lanes_max<64>(top);
    if ((threadIdx.x & 63) == 0) top4[threadIdx.x >> 6] = top;
    __syncthreads();
    const int E = unit_exponent(fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])));
    const float unit = power_of_two(6 - E), limit = 127.f * power_of_two(E - 6);
    if (mine) {
        int s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            if (i * per < a.BK)
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += round8_bits(x[i][e], unit, limit) - ROUND_BITS;
#pragma unroll
        for (int e = 0; e < 8; ++e) atomicAdd(&part[u * 8 + e], s[e]);
    }
    __syncthreads();
    const int v = (int)threadIdx.x < a.D ? part[threadIdx.x] : 0;
    const int peak = lanes_max<64>(abs(v));
    if ((threadIdx.x & 63) == 0) peak4[threadIdx.x >> 6] = peak;
    __syncthreads();
    const int shift = sum_shift(max(max(peak4[0], peak4[1]), max(peak4[2], peak4[3])));
    const int64_t at = (int64_t)bg * a.nb + j;
    if ((int)threadIdx.x < a.D) sums[at * a.D + threadIdx.x] = (int8_t)(round8_bits((float)v, power_of_two(-shift), 127.f * power_of_two(shift)) - ROUND_BITS);
    if (threadIdx.x == 0) scales[at] = power_of_two(E - 6 + shift);
}

// ---- a query in 8 bits: the sixteen lanes of a query hold eight components each (lane c: 8c ..), HB of its R heads at a time.  Every
// lane loads (one without a query or components of its own reads others'), so that the loads of several queries are on their way
// together.
template <typename T, int HB>
struct Query8 {
    const T* base;
    int64_t sh;
    int R;
    bool mine;
    Operand<T> raw[HB];
    __device__ Query8() {}
    __device__ Query8(const AttentionArgs& a, const Heads<const T>& q, int b, int t, int g, int c, bool there) : sh(q.sh), R(a.R), mine(there && c * 8 < a.D) {
        base = q.at(b, there ? t : 0, g * a.R) + min(c * 8, a.D - 8);
        fetch(0);
    }
    __device__ void fetch(int h0) {
#pragma unroll
        for (int i = 0; i < HB; ++i) raw[i] = load_operand(base + min(h0 + i, R - 1) * sh);
    }
    __device__ uint2 value() {
        float top = 0.f, x[8];
        for (int h = 0; h < R; h += HB) {
            if (h > 0) fetch(h);
#pragma unroll
            for (int i = 0; i < HB; ++i) {                     // (heads past the last are the last one again)
                numbers(raw[i], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
            }
        }
        const int E = unit_exponent(lanes_max<16>(mine ? top : 0.f));
        const float unit = power_of_two(6 - E), most = 127.f * power_of_two(E - 6);
        uint32_t s[8];                                         // (modulo 2^32)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = 0u - (uint32_t)R * (uint32_t)ROUND_BITS;
        for (int h = 0; h < R; h += HB) {
            if (R > HB) fetch(h);
#pragma unroll
            for (int i = 0; i < HB; ++i)
                if (h + i < R) {
                    numbers(raw[i], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += (uint32_t)round8_bits(x[e], unit, most);
                }
        }
        int peak = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) peak = max(peak, abs((int)s[e]));
        const int shift = sum_shift(lanes_max<16>(mine ? peak : 0));
        const float back = power_of_two(-shift), limit = 127.f * power_of_two(shift);
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2] |= (uint32_t)(round8_bits((float)(int)s[e], back, limit) & 255) << (8 * (e & 3));
        return mine ? make_uint2(w[0], w[1]) : make_uint2(0, 0);
    }
};

// ---- selection, a wavefront per 16 queries.  The 8-bit matrix instructions give the scores of 16 blocks at a time, four of them
// to each of a query's four lanes, which keeps the KK highest of its own in order: one median a place.  The four lists are
// merged; with the lowest score that is taken known, a second walk over the scores takes the blocks above it and,
// on a tie, the first that are due, in ascending order.  Summaries go through LDS, 64 blocks at a time for the workgroup's 64
// queries; the scores of up to 256 blocks stay in registers for the second walk (HELD), of more are formed again.
typedef int intx4 __attribute__((ext_vector_type(4)));
// the KK highest of the lists of lanes APART from each other, in order; the lists descend
template <int KK, int APART>
__device__ inline void merge_best(float (&x)[KK]) {
    float y[KK], z[KK];
#pragma unroll
    for (int e = 0; e < KK; ++e) {
        const Both b = both_lanes<APART>(__float_as_uint(x[e]));
        y[e] = __uint_as_float(b.first), z[KK - 1 - e] = __uint_as_float(b.second);
    }
#pragma unroll
    for (int e = 0; e < KK; ++e) x[e] = fmaxf(y[e], z[e]);     // first up, then down (or the other way round)
#pragma unroll
    for (int d = KK / 2; d >= 1; d >>= 1)
#pragma unroll
        for (int e = 0; e < KK; ++e)
            if (!(e & d)) {
                const float hi = fmaxf(x[e], x[e + d]), lo = fminf(x[e], x[e + d]);
                x[e] = hi, x[e + d] = lo;
            }
}
// Measured, 8192 queries of 20 heads over 128 blocks: 36.2 us, 42.6 with the scores formed again; HB = 4 heads at a time 40.2.  16384 queries of 32 heads
// with 8 key heads over 256 blocks: 63.5 us, 70.5 with the scores formed again; HB = 1 71.0.  Bound by the vector instructions: 8-bit queries, insertions,
// merges (the matrix instructions are busy in about 1 % of the clocks).
constexpr int SELECT_THREADS = 256, SELECT_CHUNK = 64, SELECT_HELD = 256;
template <typename T, int KK, int HB, bool HELD>
__global__ __launch_bounds__(SELECT_THREADS) void k_block_select(AttentionArgs a, Heads<const T> q, const int8_t* __restrict__ sums,
                                                                 const float* __restrict__ scales, int* __restrict__ blocks) {
    __shared__ __align__(16) uint2 q8_all[SELECT_THREADS / 64][16][17];    // a query's 128 components; 8 bytes of padding
    __shared__ __align__(16) uint2 rows[SELECT_CHUNK][17];                 // summaries likewise
    __shared__ __align__(16) float units[SELECT_CHUNK];
    const int bg = blockIdx.y, b = bg / a.G, g = bg % a.G, len = a.length(b);
    const int lane = threadIdx.x & 63, i = lane & 15, quad = lane >> 4, t0 = blockIdx.x * (SELECT_THREADS / 4) + (threadIdx.x >> 6) * 16;
    uint2(*q8)[17] = q8_all[threadIdx.x >> 6];
    const int wanted = a.NS - 1;
    const int last_p = len - a.Tq + min((int)(blockIdx.x + 1) * (SELECT_THREADS / 4), a.Tq) - 1;
    const int most = wanted > 0 && last_p >= 0 ? last_p / a.BK : 0;        // candidates of the workgroup's last query
    // 8 D / 8 pieces of eight bytes of 64 rows that lie one behind the other, four a thread at most; past the candidates the last piece again
    const int pieces = a.D / 8;
    const uint2* from = reinterpret_cast<const uint2*>(sums + (int64_t)bg * a.nb * a.D);
    const float* scl = scales + (int64_t)bg * a.nb;
    uint2 staged[4];
    float staged_unit = 0.f;
    auto fetch = [&](int j0) {
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const int u = n * SELECT_THREADS + (int)threadIdx.x;
            if (n * SELECT_THREADS < SELECT_CHUNK * pieces) staged[n] = from[min(j0 * pieces + u, most * pieces - 1)];
        }
        staged_unit = scl[min(j0 + (int)threadIdx.x % SELECT_CHUNK, most - 1)];
    };
    auto put = [&]() {
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const int u = n * SELECT_THREADS + (int)threadIdx.x;
            if (u < SELECT_CHUNK * pieces) rows[u / pieces][u % pieces] = staged[n];
        }
        if (threadIdx.x < SELECT_CHUNK) units[threadIdx.x] = staged_unit;
    };
    if (most > 0) fetch(0);
    for (int u = threadIdx.x; u < SELECT_CHUNK * 17; u += SELECT_THREADS) rows[0][u] = make_uint2(0, 0);
    {
        Query8<T, HB> queries[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int tq = t0 + r * 4 + quad;
            queries[r] = Query8<T, HB>(a, q, b, tq, g, i, tq < a.Tq && len - a.Tq + tq >= 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) q8[r * 4 + quad][i] = queries[r].value();
    }
    __syncthreads();
    intx4 qb[2];                                               // column = query, 16 components of every 64 to a lane
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const uint2 lo = q8[i][c * 8 + quad * 2], hi = q8[i][c * 8 + quad * 2 + 1];
        qb[c] = intx4{(int)lo.x, (int)lo.y, (int)hi.x, (int)hi.y};
    }
    const int t = t0 + i, p = len - a.Tq + t;
    const bool there = t < a.Tq && p >= 0;
    const int mine = there ? p / a.BK : 0;                     // candidates: the blocks before it
    auto scores = [&](int j0, int at, float* v) {              // of the blocks j0 + 4 quad + r, which lie at `at` of the chunk
        intx4 c = {0, 0, 0, 0}, ab;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (h * 64 < a.D) {
                const uint2 lo = rows[at + i][h * 8 + quad * 2], hi = rows[at + i][h * 8 + quad * 2 + 1];
                ab = intx4{(int)lo.x, (int)lo.y, (int)hi.x, (int)hi.y};
                c = __builtin_amdgcn_mfma_i32_16x16x64_i8(ab, qb[h], c, 0, 0, 0);
            }
        const float4 u = *reinterpret_cast<const float4*>(&units[at + 4 * quad]);
        const float unit[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = j0 + 4 * quad + r < mine ? (float)c[r] * unit[r] : -INFINITY;
    };
    float best[KK];                                            // descending
#pragma unroll
    for (int e = 0; e < KK; ++e) best[e] = -INFINITY;
    auto insert = [&](const float* v) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (__any(v[r] > best[KK - 1])) {
#pragma unroll
                for (int e = KK - 1; e > 0; --e) best[e] = __builtin_amdgcn_fmed3f(v[r], best[e - 1], best[e]);
                best[0] = fmaxf(v[r], best[0]);
            }
    };
    float held[HELD ? SELECT_HELD / 4 : 4];
    constexpr int CHUNKS = HELD ? SELECT_HELD / SELECT_CHUNK : 1;
    auto chunk_in = [&](int j0, bool again) {                  // the chunk to LDS, the next one on its way
        __syncthreads();
        put();
        __syncthreads();
        if (j0 + SELECT_CHUNK < most) fetch(j0 + SELECT_CHUNK);
        else if (again) fetch(0);
    };
    if constexpr (HELD) {
#pragma unroll
        for (int n = 0; n < CHUNKS; ++n)
            if (n * SELECT_CHUNK < most) {
                chunk_in(n * SELECT_CHUNK, false);
#pragma unroll
                for (int s = 0; s < SELECT_CHUNK / 16; ++s)
                    if (n * SELECT_CHUNK + s * 16 < most) {
                        scores(n * SELECT_CHUNK + s * 16, s * 16, held + n * 16 + s * 4);
                        insert(held + n * 16 + s * 4);
                    }
            }
    } else {
        for (int j0 = 0; j0 < most; j0 += SELECT_CHUNK) {
            chunk_in(j0, true);
            for (int s = 0; s < SELECT_CHUNK && j0 + s < most; s += 16) {
                scores(j0 + s, s, held);
                insert(held);
            }
        }
    }
    merge_best<KK, 16>(best);
    merge_best<KK, 32>(best);
    float least = -INFINITY;                                   // the lowest that is taken
#pragma unroll
    for (int e = 0; e < KK; ++e)
        if (e == wanted - 1) least = best[e];
    int due = 0;                                               // how many equal to it are taken
#pragma unroll
    for (int e = 0; e < KK; ++e) due += (e < wanted && best[e] == least) ? 1 : 0;
    int* out = blocks + ((int64_t)bg * a.Tq + t) * a.NS;
    int n_out = 0;
    auto take = [&](int j0, const float* v) {
        uint32_t both = 0;                                     // bits of the query's sixteen blocks: above, equal
#pragma unroll
        for (int r = 0; r < 4; ++r) both |= (v[r] > least ? 1u : v[r] == least && v[r] > -INFINITY ? 0x10000u : 0u) << r;
        both <<= 4 * quad;
        both = apart<16>(both, [](uint32_t x, uint32_t y) { return x | y; });
        both = apart<32>(both, [](uint32_t x, uint32_t y) { return x | y; });
        uint32_t above = both & 0xFFFF, equal = both >> 16;
        while (__popc(equal) > due) equal &= ~(1u << (31 - __clz(equal)));
        due -= __popc(equal);
        above |= equal;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int bit = 4 * quad + r;
            if (above >> bit & 1) out[n_out + __popc(above & ((1u << bit) - 1))] = j0 + bit;
        }
        n_out += __popc(above);
    };
    if constexpr (HELD) {
#pragma unroll
        for (int n = 0; n < SELECT_HELD / 16; ++n)
            if (n * 16 < most) take(n * 16, held + n * 4);
    } else {
        for (int j0 = 0; j0 < most; j0 += SELECT_CHUNK) {
            chunk_in(j0, false);
            for (int s = 0; s < SELECT_CHUNK && j0 + s < most; s += 16) {
                scores(j0 + s, s, held);
                take(j0 + s, held);
            }
        }
    }
    if (t < a.Tq)
        for (int e = n_out + quad; e < a.NS; e += 4) out[e] = e == n_out && there ? mine : -1;
}

// ---- selection for few queries: a workgroup per query and key head.  Every thread scores blocks; then one wavefront takes the scores
// to registers, U a lane, finds the lowest that is taken bit by bit, counting the scores at or above a trial value in its lane
// masks, and writes the blocks in order: no barrier in 32 steps.
constexpr int FEW_THREADS = 256;
// scores as unsigned numbers of the same order, above 0
__device__ inline uint32_t ordered(float x) {
    x += 0.f;                                                  // -0 and +0 are one score
    const uint32_t u = __float_as_uint(x);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
template <int U>
__device__ inline void take_best(const uint32_t* score, int candidates, int wanted, int own, int NS, int* __restrict__ out) {
    const int lane = threadIdx.x;
    uint32_t v[U];                                             // block u 64 + lane; 0: none
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = u * 64 + lane < candidates ? score[u * 64 + lane] : 0u;
    uint32_t least = 0;                                        // the highest value with at least `wanted` scores at or above it
    int at_least = candidates;
    if (wanted < candidates)
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t trial = least | (1u << bit);
            int c = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) c += __popcll(__ballot(v[u] >= trial));
            if (c >= wanted) least = trial, at_least = c;
            if (c == wanted) break;
        }
    int equal = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) equal += __popcll(__ballot(v[u] == least && v[u] != 0));
    int due = wanted - (at_least - equal), n = 0;              // of the equal ones, the first so many
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t below = (1ull << lane) - 1, same = __ballot(v[u] == least && v[u] != 0);
        const bool take = v[u] > least || ((same >> lane & 1) && __popcll(same & below) < due);
        const uint64_t all = __ballot(take);
        if (take) out[n + __popcll(all & below)] = u * 64 + lane;
        n += __popcll(all);
        due -= min(due, (int)__popcll(same));
    }
    for (int i = n + lane; i < NS; i += 64) out[i] = i == n ? own : -1;
}
template <typename T>
__global__ __launch_bounds__(FEW_THREADS) void k_block_select_few(AttentionArgs a, Heads<const T> q, const int8_t* __restrict__ sums,
                                                                  const float* __restrict__ scales, int* __restrict__ blocks) {
    __shared__ __align__(16) uint2 q8[16];
    __shared__ uint32_t score[KEY_BLOCKS_MAX];
    const int bg = blockIdx.y, b = bg / a.G, g = bg % a.G, len = a.length(b), t = blockIdx.x;
    const int p = len - a.Tq + t;
    int* out = blocks + ((int64_t)bg * a.Tq + t) * a.NS;
    if (p < 0) {
        for (int n = threadIdx.x; n < a.NS; n += FEW_THREADS) out[n] = -1;
        return;
    }
    const int own = p / a.BK, wanted = min(a.NS - 1, own);
    if (threadIdx.x < 64) {
        const uint2 w = Query8<T, 4>(a, q, b, t, g, threadIdx.x & 15, true).value();
        if (threadIdx.x < 16) q8[threadIdx.x] = w;
    }
    __syncthreads();
    const int8_t* srow = sums + (int64_t)bg * a.nb * a.D;
    const float* scl = scales + (int64_t)bg * a.nb;
    if (wanted > 0)
        for (int j = threadIdx.x; j < own; j += FEW_THREADS) {
            const uint2* s = reinterpret_cast<const uint2*>(srow + (int64_t)j * a.D);
            int dot = 0;
#pragma unroll 4
            for (int u = 0; u < a.D / 8; ++u) {
                const uint2 w = s[u], x = q8[u];
                dot = __builtin_amdgcn_sdot4((int)w.x, (int)x.x, dot, false);
                dot = __builtin_amdgcn_sdot4((int)w.y, (int)x.y, dot, false);
            }
            score[j] = ordered((float)dot * scl[j]);
        }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const int candidates = wanted > 0 ? own : 0;
    if (candidates <= 256) take_best<4>(score, candidates, wanted, own, a.NS, out);
    else if (candidates <= 1024) take_best<16>(score, candidates, wanted, own, a.NS, out);
    else take_best<32>(score, candidates, wanted, own, a.NS, out);
}

// ---- plan: the entries of a selection that count, in order.  Selections go through LDS, from and to memory in order.
constexpr int PLAN_ROWS = 256;           // queries of a workgroup
__device__ inline void rows_to_lds(const AttentionArgs& a, const int* __restrict__ from, int n, int* rows) {
    for (int i = threadIdx.x; i < n * a.NS; i += PLAN_ROWS) rows[i / a.NS * (a.NS | 1) + i % a.NS] = from[i];      // (odd rows: a thread each, in different banks)
}
__global__ __launch_bounds__(PLAN_ROWS) void k_plan_rows(AttentionArgs a, const int* __restrict__ blocks, Plan plan) {
    extern __shared__ __align__(16) char lds[];
    int* rows = reinterpret_cast<int*>(lds);
    const int bg = blockIdx.y, t0 = blockIdx.x * PLAN_ROWS, n = min(PLAN_ROWS, a.Tq - t0);
    const int64_t first = ((int64_t)bg * a.Tq + t0) * a.NS;
    rows_to_lds(a, blocks + first, n, rows);
    __syncthreads();
    if ((int)threadIdx.x < n) {
        const int p = a.length(bg / a.G) - a.Tq + t0 + (int)threadIdx.x, own = p >= 0 ? p / a.BK : -1;
        int* row = rows + threadIdx.x * (a.NS | 1);
        int last = -1, kept = 0;
        for (int s = 0; s < a.NS; ++s) {
            const int j = row[s];
            if (j > last && j <= own) row[kept++] = last = j;
        }
        for (; kept < a.NS; ++kept) row[kept] = a.nb;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n * a.NS; i += PLAN_ROWS) plan.rows[first + i] = rows[i / a.NS * (a.NS | 1) + i % a.NS];
}

// ---- lists.  A tile of 256 queries marks its queries in one bit word of 256 a block: a query has a block once at most, so the number
// of bits below its own is its place among the tile's.  Counts per tile, their sums over the tiles, then every pair to its place: 9, 7 and 13 us
// for 8192 queries of 20 key heads with 8 blocks (latency, and scattered writes of 5 MB).
struct ListSpace {
    int bits, rows, total;               // LDS: [nb][8] words, [256][NS + 1]
    ListSpace(const AttentionArgs& a) : bits(0), rows(a.nb * 32), total(a.nb * 32 + LIST_TILE * (a.NS | 1) * 4) {}
};
__device__ inline void mark_tile(const AttentionArgs& a, const int* __restrict__ from, int n, uint32_t* bits, int* rows) {
    for (int i = threadIdx.x; i < a.nb * 8; i += LIST_TILE) bits[i] = 0;
    rows_to_lds(a, from, n, rows);
    __syncthreads();
    const int* row = rows + threadIdx.x * (a.NS | 1);
    if ((int)threadIdx.x < n)
        for (int s = 0; s < a.NS && row[s] < a.nb; ++s) atomicOr(&bits[row[s] * 8 + (threadIdx.x >> 5)], 1u << (threadIdx.x & 31));
    __syncthreads();
}
__global__ __launch_bounds__(LIST_TILE) void k_list_count(AttentionArgs a, Plan plan, Lists lists, int bg0, ListSpace space) {
    extern __shared__ __align__(16) char lds[];
    uint32_t* bits = reinterpret_cast<uint32_t*>(lds + space.bits);
    const int gg = blockIdx.y, t0 = blockIdx.x * LIST_TILE;
    mark_tile(a, plan.rows + ((int64_t)(bg0 + gg) * a.Tq + t0) * a.NS, min(LIST_TILE, a.Tq - t0), bits, reinterpret_cast<int*>(lds + space.rows));
    int* counts = lists.tile + ((int64_t)gg * lists.tiles + blockIdx.x) * a.nb;
    for (int j = threadIdx.x; j < a.nb; j += LIST_TILE) {
        int c = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) c += __popc(bits[j * 8 + w]);
        counts[j] = c;
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

// a workgroup per (batch, key head): `width` blocks at a time, 1024 / width stretches of the tiles side by side
__global__ __launch_bounds__(1024) void k_list_sums(AttentionArgs a, Lists lists, int width) {
    __shared__ int stretch_sum[1024];
    const int gg = blockIdx.x, stretches = 1024 / width, mine = threadIdx.x / width;
    const int i0 = (int)((int64_t)lists.tiles * mine / stretches), i1 = (int)((int64_t)lists.tiles * (mine + 1) / stretches);
    int* tile = lists.tile + (int64_t)gg * lists.tiles * a.nb;
    int* start = lists.start + (int64_t)gg * (a.nb + 1);
    int* item_start = lists.item_start + (int64_t)gg * (a.nb + 1);
    int2* items = lists.items + (int64_t)gg * lists.max_items;
    int2 done = make_int2(0, 0);
    for (int j0 = 0; j0 < a.nb; j0 += width) {
        const int j = j0 + (int)(threadIdx.x % width);
        const bool there = j < a.nb;
        int n = 0;
        if (there)
#pragma unroll 8
            for (int i = i0; i < i1; ++i) n += tile[(int64_t)i * a.nb + j];
        stretch_sum[threadIdx.x] = n;
        __syncthreads();
        int before = 0, whole = 0;
        for (int s = 0; s < stretches; ++s) {
            const int c = stretch_sum[s * width + threadIdx.x % width];
            before += s < mine ? c : 0;
            whole += c;
        }
        if (there)
#pragma unroll 8
            for (int i = i0; i < i1; ++i) {
                const int c = tile[(int64_t)i * a.nb + j];
                tile[(int64_t)i * a.nb + j] = before;
                before += c;
            }
        const int pairs = there && mine == 0 ? whole : 0, parts = (pairs + lists.item_pairs - 1) / lists.item_pairs;
        int2 all;
        const int2 at = exclusive(make_int2(pairs, parts), &all);          // (the threads of the first stretch come first)
        if (there && mine == 0) {
            start[j] = done.x + at.x;
            item_start[j] = done.y + at.y;
            for (int i = 0; i < parts; ++i) items[done.y + at.y + i] = make_int2(j, done.x + at.x + i * lists.item_pairs);
        }
        done.x += all.x, done.y += all.y;
    }
    if (threadIdx.x == 0) start[a.nb] = done.x, item_start[a.nb] = done.y;
}

__global__ __launch_bounds__(LIST_TILE) void k_list_fill(AttentionArgs a, Plan plan, Lists lists, int bg0, ListSpace space) {
    extern __shared__ __align__(16) char lds[];
    uint32_t* bits = reinterpret_cast<uint32_t*>(lds + space.bits);
    int* rows = reinterpret_cast<int*>(lds + space.rows);
    const int gg = blockIdx.y, t0 = blockIdx.x * LIST_TILE, n = min(LIST_TILE, a.Tq - t0), word = threadIdx.x >> 5;
    mark_tile(a, plan.rows + ((int64_t)(bg0 + gg) * a.Tq + t0) * a.NS, n, bits, rows);
    if ((int)threadIdx.x >= n) return;
    const int* row = rows + threadIdx.x * (a.NS | 1);
    const int* before = lists.tile + ((int64_t)gg * lists.tiles + blockIdx.x) * a.nb;
    const int* start = lists.start + (int64_t)gg * (a.nb + 1);
    int* list = lists.list + (int64_t)gg * a.Tq * a.NS;
    for (int s = 0; s < a.NS && row[s] < a.nb; ++s) {
        const int j = row[s];
        int at = start[j] + before[j] + __popc(bits[j * 8 + word] & ((1u << (threadIdx.x & 31)) - 1));
        for (int w = 0; w < word; ++w) at += __popc(bits[j * 8 + w]);
        list[at] = (t0 + (int)threadIdx.x) << SELECT_BITS | s;
    }
}

// Single tokens, and fewer (query, key head) than this: a workgroup for each.  The other kernel walks the summaries one chunk after the other, 64 queries of a
// key head together, and leaves most of the card idle until there are many.  Kernel times, each query's own workgroup against the other, heads of 128 with four to
// a key head: single tokens of 128 x 8 key heads, 16, 64, 256 and 1024 blocks: 7, 9, 14 and 37 us against 16, 19, 33 and 94; of 512 x 8: 22, 35, 45 and 151
// against 49, 58, 105 and 353 (one head of 64 each, 4 selected, 384 x 12, 16 blocks, the closest: 28 against 30).  Two queries of 384 x 12 with such heads: 54 against 31.
// Eight of 16 x 8 (1024), 16, 64, 256 blocks: 7, 10, 13 against 8, 10, 20; sixteen (2048): 12, 17, 23 against 8, 10, 20.
constexpr int FEW_QUERIES = 1024;

}  // namespace

int build_lists(const AttentionArgs& a, const Plan& plan, const Lists& lists, int bg0, int n, hipStream_t st) {
    const dim3 grid((unsigned)lists.tiles, (unsigned)n);
    const ListSpace space(a);                                   // 129 KB at most
    static uint64_t allowed_count = 0, allowed_fill = 0;
    if (space.total > 64 * 1024) {
        if (int e = allow_lds(reinterpret_cast<const void*>(&k_list_count), LDS_BYTES, allowed_count)) return e;
        if (int e = allow_lds(reinterpret_cast<const void*>(&k_list_fill), LDS_BYTES, allowed_fill)) return e;
    }
    if (lists.tiles > 0) {
        k_list_count<<<grid, LIST_TILE, space.total, st>>>(a, plan, lists, bg0, space);
        MST_LAUNCH_CHECK();
    }
    int width = 16;                                             // blocks that the threads of the sums stand for: a power of two
    while (width < a.nb && width < 1024) width *= 2;
    k_list_sums<<<(unsigned)n, 1024, 0, st>>>(a, lists, width);
    MST_LAUNCH_CHECK();
    if (lists.tiles > 0) {
        k_list_fill<<<grid, LIST_TILE, space.total, st>>>(a, plan, lists, bg0, space);
        MST_LAUNCH_CHECK();
    }
    return MST_OK;
}

}  // namespace mst

extern "C" int mst_key_summary(const mst_attention_shape* s, const mst_heads* k, int8_t* sums, float* scales, int new_tokens, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    if (new_tokens < 0) return MST_ERR_ARG;
    // blocks that a sequence's last new_tokens keys can complete
    const int64_t most = new_tokens == 0 ? 0 : std::min<int64_t>(s->keys / s->block, (int64_t)new_tokens / s->block + 1);
    if (s->batch == 0 || most == 0) return MST_OK;             // (buffers may be null)
    if (!sums || !scales || !aligned16(sums) || !aligned16(scales)) return MST_ERR_ARG;
    if (int e = check_heads(k, s->batch, s->keys, s->kv_heads, s->type, false)) return e;
    const AttentionArgs a = attention_args(s);
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
    if (s->batch == 0 || s->queries == 0) return MST_OK;
    if ((s->keys > 0 && (!sums || !scales)) || !blocks || !aligned16(sums) || !aligned16(scales) || !aligned16(blocks)) return MST_ERR_ARG;
    if (int e = check_heads(q, s->batch, s->queries, s->heads, s->type, false)) return e;
    const AttentionArgs a = attention_args(s);
    hipStream_t st = static_cast<hipStream_t>(stream);
    with_type(s->type, [&](auto t) {
        using T = decltype(t);
        const Heads<const T> qh = heads_of<const T>(q);
        if (a.Tq == 1 || (int64_t)a.Tq * a.B * a.G < FEW_QUERIES) {
            k_block_select_few<T><<<dim3((unsigned)a.Tq, (unsigned)(a.B * a.G)), FEW_THREADS, 0, st>>>(a, qh, sums, scales, blocks);
            return;
        }
        const dim3 grid((unsigned)cdiv(a.Tq, SELECT_THREADS / 4), (unsigned)(a.B * a.G));
        const int wanted = a.NS - 1;
        auto launch = [&](auto kk) {
            constexpr int KK = decltype(kk)::value;
            auto go = [&](auto hb, auto held) { k_block_select<T, KK, decltype(hb)::value, decltype(held)::value><<<grid, SELECT_THREADS, 0, st>>>(a, qh, sums, scales, blocks); };
            auto heads = [&](auto held) {
                if (a.R == 1) go(std::integral_constant<int, 1>{}, held);
                else go(std::integral_constant<int, 4>{}, held);
            };
            if (a.nb <= SELECT_HELD) heads(std::true_type{});
            else heads(std::false_type{});
        };
        if (wanted <= 4) launch(std::integral_constant<int, 4>{});
        else if (wanted <= 8) launch(std::integral_constant<int, 8>{});
        else if (wanted <= 16) launch(std::integral_constant<int, 16>{});
        else if (wanted <= 32) launch(std::integral_constant<int, 32>{});
        else launch(std::integral_constant<int, 64>{});
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
    if (s->batch == 0 || s->queries == 0) return MST_OK;
    if (!blocks || !plan_dev || !aligned16(blocks) || !aligned16(plan_dev)) return MST_ERR_ARG;
    const AttentionArgs a = attention_args(s);
    const Plan plan = carve_plan(plan_dev, a);
    if (plan_bytes < plan.total) return MST_ERR_WORKSPACE;
    const size_t lds = (size_t)PLAN_ROWS * (a.NS | 1) * 4;      // 65 KB at most
    static uint64_t allowed = 0;
    if (lds > 64 * 1024)
        if (int e = allow_lds(reinterpret_cast<const void*>(&k_plan_rows), LDS_BYTES, allowed)) return e;
    k_plan_rows<<<dim3((unsigned)cdiv(a.Tq, PLAN_ROWS), (unsigned)(a.B * a.G)), PLAN_ROWS, lds, static_cast<hipStream_t>(stream)>>>(a, blocks, plan);
    MST_LAUNCH_CHECK();
    return MST_OK;
}
