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

// LDS position of unit u (eight k) of row m of an operand along: the sixteen rows of a read cover all banks
__device__ __forceinline__ uint32_t along_unit(int m, int u) {
    const int rho = (m & ~15) | ((m & 3) << 2) | ((m >> 2) & 3);
    return (uint32_t)(rho * 64 + (((u ^ (rho >> 2)) & 3) << 4));
}
// The 32-byte units (16 columns) of row k of an operand across are kept at unit ^ swizzle(k): so do the eight rows of half a wavefront
__device__ __forceinline__ int across_swizzle(int k) { return (k & 3) | ((k >> 1) & 4); }

enum Epilogue { STATS, LOGIT_GRAD, LOGIT_GRAD_PARTS, SUMS, OUT_F32, OUT_BF16 };
template <Epilogue E> struct EpilogueArgs;
template <> struct EpilogueArgs<STATS> { using type = VocabStats; };
template <int PLANES> struct VocabLogitGradOf : VocabLogitGrad {};
template <> struct EpilogueArgs<LOGIT_GRAD> { using type = VocabLogitGradOf<1>; };
template <> struct EpilogueArgs<LOGIT_GRAD_PARTS> { using type = VocabLogitGradOf<PLANES_MAX>; };
template <> struct EpilogueArgs<SUMS> { using type = VocabSums; };
template <typename T> struct VocabOutOf : VocabOut {};
template <> struct EpilogueArgs<OUT_F32> { using type = VocabOutOf<float>; };
template <> struct EpilogueArgs<OUT_BF16> { using type = VocabOutOf<bf16>; };

// Results: acc[i][j][v] is row m0 + 16 i + lane % 16, column n0 + 16 j + 4 (lane / 16) + v of C; a wavefront's 16 I rows and 16 J columns.
// Results go straight to memory: a store writes 32 or 64 bytes of sixteen rows, and those that fill a line follow one another.  (Through LDS, in whole lines, they
// waited longer than they saved.)
// Result v of a 16 x 16 product: it lies in accumulation registers and is read out where it is used (left to the compiler, most of them are read at once, and other
// registers spill).
__device__ __forceinline__ float result(const floatx4& acc, int v) {
    float x;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(acc[v]));
    return x;
}

// ... or of two sums
struct TwoSums { floatx4 main, low; };
__device__ __forceinline__ float result(const TwoSums& acc, int v) { return result(acc.main, v) + result(acc.low, v); }
__device__ __forceinline__ void clear_sum(floatx4& acc) { acc = floatx4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ void clear_sum(TwoSums& acc) { acc.main = acc.low = floatx4{0.f, 0.f, 0.f, 0.f}; }
// What a vector instruction has written into it is two wait states away from the matrix instructions behind, once all are held and settle() has followed.
__device__ __forceinline__ void hold_sum(floatx4& acc) { asm volatile("" : "+a"(acc)); }
__device__ __forceinline__ void hold_sum(TwoSums& acc) { asm volatile("" : "+a"(acc.main), "+a"(acc.low)); }
__device__ __forceinline__ void settle() { asm volatile("s_nop 1"); }

// Sums of exp2(z log2 e - base) over a wavefront's columns, those below p.n.  Base is the logit of the row's own label: the sum over all columns is then 1 at least,
// what is lost below fp32 does not count in it, and no maximum has to be found first (a fifth of the instructions).  A sum that passes 2^64 (or is no number) is formed
// again from the row's maximum here.  A row's sums, 2^18 at most, are added elsewhere: those with the label's base stay below 2^82 together, and what falls below fp32 of them beside a sum
// with another base, 1 at least in its own, is less than 2^(64 - 126 + 18) of that.
constexpr float SUM_MOST = 0x1p64f;
template <int I, int J, bool ENDS, bool MAXIMUM, typename X>
__device__ __forceinline__ bool statistics(const VocabStats& e, const VocabProduct& p, const X (&acc)[I][J], int m0, int n0, int lane) {
    const int last = p.n - n0 - 4 * (lane >> 4);
    auto larger = [](float a, float b) { return fmaxf(a, b); };
    auto plus = [](float a, float b) { return a + b; };
    float2* const to = e.stats + (int64_t)(e.first + n0 / (16 * J)) * e.row_stride + m0 + (lane & 15);
    float base[I];
#pragma unroll
    for (int i = 0; i < I; ++i) base[i] = MAXIMUM ? 0.f : e.at_label[m0 + 16 * i + (lane & 15)] * LOG2E;
    bool fits = true;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        auto z = [&](int j, int v) __attribute__((always_inline)) {
            const float x = result(acc[i][j], v);
            return !ENDS || 16 * j + v < last ? x : -INFINITY;
        };
        if constexpr (MAXIMUM) {
            float top = z(0, 0);
#pragma unroll
            for (int j = 0; j < J; ++j) top = fmaxf(fmaxf(fmaxf(top, z(j, 0)), fmaxf(z(j, 1), z(j, 2))), z(j, 3));
            base[i] = apart<32>(apart<16>(top, larger), larger) * LOG2E;
        }
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) sum += exp2_fast(fmaf(z(j, v), LOG2E, -base[i]));
        sum = apart<32>(apart<16>(sum, plus), plus);
        fits &= sum < SUM_MOST;
        if (lane < 16) to[16 * i] = make_float2(base[i], sum);
        __builtin_amdgcn_sched_barrier(0);                          // (with the results of several rows out of the accumulation registers it spills)
    }
    return fits;
}
template <int I, int J, bool ENDS, typename X>
__device__ __forceinline__ void statistics(const VocabStats& e, const VocabProduct& p, const X (&acc)[I][J], int m0, int n0, int lane) {
    if (__any(!statistics<I, J, ENDS, false>(e, p, acc, m0, n0, lane))) statistics<I, J, ENDS, true>(e, p, acc, m0, n0, lane);
}
template <int I, int J, typename X>
__device__ __forceinline__ void finish(const VocabStats& e, const VocabProduct& p, X (&acc)[I][J], int m0, int n0, int, int lane, int) {
    if (n0 + 16 * J <= p.n) statistics<I, J, false>(e, p, acc, m0, n0, lane);
    else if (n0 < p.n) statistics<I, J, true>(e, p, acc, m0, n0, lane);
}

// dz
template <int I, int J, int PLANES, bool ENDS, typename X>
__device__ __forceinline__ void logit_grad(const VocabLogitGrad& e, const VocabProduct& p, const X (&acc)[I][J], int m0, int n0, int lane) {
    const int g = lane >> 4, last = p.n - n0 - 4 * g;
    float base[I], d[I], at_label[I];
    int label[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int m = m0 + 16 * i + (lane & 15);
        const float lse = e.lse[m];
        base[i] = lse * LOG2E;
        // What the product's rounding loses (1e-6 of a row's dz where its lse is 20) is made up for in d: its own exact remainder.  (Rows of no token: infinite - infinite.)
        const float left = fmaf(lse, LOG2E, -base[i]);
        d[i] = e.d[m] * (lse < INFINITY ? exp2_fast(-left) : 1.f);
        at_label[i] = e.at_label[m];
        label[i] = e.label[m] - e.v0 - n0;
    }
#pragma unroll
    for (int i = 0; i < I; ++i) {
        uint16_t* const row = e.ds + (int64_t)(m0 + 16 * i + (lane & 15)) * e.ld + n0 + 4 * g;
        auto put = [&](auto labels) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                float x[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    x[v] = d[i] * exp2_fast(fmaf(result(acc[i][j], v), LOG2E, -base[i]));
                    if (ENDS) x[v] = 16 * j + v < last ? x[v] : 0.f;
                    if (decltype(labels)::value && 16 * j + 4 * g + v == label[i]) x[v] = at_label[i];
                }
#pragma unroll
                for (int part = 0; part < PLANES; ++part) {
                    const uint32_t a = pack2(x[0], x[1]), b = pack2(x[2], x[3]);
                    *reinterpret_cast<uint2*>(row + part * e.plane + 16 * j) = make_uint2(a, b);
                    x[0] -= __uint_as_float(a << 16);
                    x[1] -= __uint_as_float(a & 0xFFFF0000u);
                    x[2] -= __uint_as_float(b << 16);
                    x[3] -= __uint_as_float(b & 0xFFFF0000u);
                }
            }
        };
        // (one in 25 has a label of its sixteen rows among these columns)
        if (__any(label[i] >= 0 && label[i] < 16 * J)) put(std::true_type{});
        else put(std::false_type{});
        __builtin_amdgcn_sched_barrier(0);
    }
}
template <int I, int J, int PLANES, typename X>
__device__ __forceinline__ void finish(const VocabLogitGradOf<PLANES>& e, const VocabProduct& p, X (&acc)[I][J], int m0, int n0, int, int lane, int) {
    if (n0 + 16 * J <= p.n) logit_grad<I, J, PLANES, false>(e, p, acc, m0, n0, lane);
    else logit_grad<I, J, PLANES, true>(e, p, acc, m0, n0, lane);
}

// Sums lie as the wavefronts hold them, a wavefront's 16 x 16 results in 1 KB after another (sum_place): the next piece begins with them.
__device__ __forceinline__ floatx4& main_sum(floatx4& acc) { return acc; }
__device__ __forceinline__ floatx4& main_sum(TwoSums& acc) { return acc.main; }
__device__ __forceinline__ floatx4 whole_sum(const floatx4& acc) { return acc; }
__device__ __forceinline__ floatx4 whole_sum(const TwoSums& acc) { return acc.main + acc.low; }
__device__ __forceinline__ float4* sums_of(const VocabSums& e, int m0, int n0, int split, int lane) {
    return reinterpret_cast<float4*>(e.sums + split * e.stride) + sum_place(m0, n0, e.wide) + lane;
}
template <int I, int J, typename X>
__device__ __forceinline__ void begin(const VocabSums& e, X (&acc)[I][J], int m0, int n0, int split, int lane) {
    if (!e.add) return;
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) main_sum(acc[i][j]) = *reinterpret_cast<const floatx4*>(sums_of(e, m0 + 16 * i, n0 + 16 * j, split, lane));
}
template <int I, int J, typename Args, typename X>
__device__ __forceinline__ void begin(const Args&, X (&)[I][J], int, int, int, int) {}
template <int I, int J, typename X>
__device__ __forceinline__ void finish(const VocabSums& e, const VocabProduct&, X (&acc)[I][J], int m0, int n0, int split, int lane, int) {
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) *reinterpret_cast<floatx4*>(sums_of(e, m0 + 16 * i, n0 + 16 * j, split, lane)) = whole_sum(acc[i][j]);
}
template <int I, int J, typename T, typename X>
__device__ __forceinline__ void finish(const VocabOutOf<T>& e, const VocabProduct& p, X (&acc)[I][J], int m0, int n0, int, int lane, int m_rows) {
    const float u = *e.unit;
    const int m = m0 + (lane & 15), n = n0 + 4 * (lane >> 4);
    T* const first = static_cast<T*>(e.out) + (int64_t)m * e.ld + n;
    auto put = [&](auto ends) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            T* const row = first + (int64_t)(16 * i) * e.ld;
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (!decltype(ends)::value || (m + 16 * i < m_rows && n + 16 * j < p.n))       // (p.n a multiple of eight)
                    store4(row + 16 * j, u * result(acc[i][j], 0), u * result(acc[i][j], 1), u * result(acc[i][j], 2), u * result(acc[i][j], 3));
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (m0 + 16 * I <= m_rows && n0 + 16 * J <= p.n) put(std::false_type{});
    else put(std::true_type{});
}

// Of the stores of a unit's results, so many are issued whatever the unit holds (dz: one a product of 16 x 16 and part; 52: as many as the counter of outstanding accesses can
// tell apart beside the loads)
constexpr int stores_behind(Epilogue E, int products) {
    const int stores = E == LOGIT_GRAD ? products : E == LOGIT_GRAD_PARTS ? PLANES_MAX * products : 0;
    return stores < 52 ? stores : 52;
}

// ---- tiles of 256 x 256, four wavefronts of 128 x 128, the sums in the accumulation half of the registers; and of 128 x 128, four of 64 x 64, two workgroups to a CU
// A stage of LDS is 64 contraction indices of one operand, 32 KB (16), so that rows of memory are read in whole lines of 128 bytes; five of them, A and B in turn.
// One wavefront a SIMD has nothing to hide behind: every step's (32 indices') operand reads, for the next step, and a stage's loads, for two to three steps
// after that, stand one by one between its 64 matrix instructions (16).  Steps come in pairs, of which the second waits for the pair behind it:
//   first   products of its first half, reads of its second half, loads of the next pair but one: A
//   second  waits; products of its second half, reads of the next pair's first half, loads of the next pair but one: B
// 8192 tokens, width 1280, vocabulary 50257 (1054 GFLOP a product): statistics 863 us, 1222 TFLOP/s; dz 1042 (two pieces), 1012; dh 894, 1180; dE 862, 1223; the library's 8192^3 product
// reaches 1191.  Matrix instructions are busy in 70 % of the clocks (dz, whose 64 stores and exponentials of a tile hide behind nothing: 56), at some 1.8 GHz.  Of 768 tokens of width 768
// 591 tiles take three rounds of the 256 CUs: statistics 69 us, 860 TFLOP/s; dz 87, dh 69, dE 84.
// What bounds the loop is the way of the loads into LDS, 64 KB a pair of steps and CU; small tiles load twice as much a product (which of them: vocab_side).  Of the whole of the above, 3.5 ms now,
// results that leave for memory and loads that begin only then took 4.46, workgroups that stay and load ahead 4.25.
constexpr int L_PAIR = 2 * VK, L_STAGES = 5;
constexpr int l_stage(int side) { return side * L_PAIR * 2; }

// The 16-byte units (eight indices) of a row of an operand along are kept at unit ^ mix(row): sixteen rows of a read cover all banks
__device__ __forceinline__ int pair_mix(int row) { return (row >> 1) & 7; }

// One operand's share of a wavefront's loads
template <bool ALONG, int SIDE>
struct TileLoads {
    static constexpr int PIECES = SIDE / 32;        // of 1 KB, a stage's
    uint32_t v[PIECES];
    const char* base;                    // of the pair
    __device__ __forceinline__ void aim_rows(const VocabOperand& o, int first, int wave, int lane, int left, int turn) {
        const uint32_t row_bytes = 2u * (uint32_t)o.ld;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int piece = PIECES * wave + (j ^ turn);
            if constexpr (ALONG) {
                const int row = 8 * piece + (lane >> 3), u = (lane & 7) ^ pair_mix(row);
                v[j] = (uint32_t)min(row, o.rows - 1 - first) * row_bytes + 16u * u;
            } else {                     // left: contraction indices from this pair on
                constexpr int WORDS = SIDE / 8;      // of 16 bytes, of a contraction index
                const int k = 64 / WORDS * piece + lane / WORDS, col = 16 * ((lane % WORDS >> 1) ^ across_swizzle(k)) + 8 * (lane & 1);
                v[j] = (uint32_t)min(k, left - 1) * row_bytes + 2u * (uint32_t)min((int64_t)col, o.ld - 8 - first);
            }
        }
    }
    __device__ __forceinline__ void aim_pair(const VocabOperand& o, int first, int t) {
        base = reinterpret_cast<const char*>(ALONG ? o.p + (int64_t)first * o.ld + t * L_PAIR : o.p + (int64_t)t * L_PAIR * o.ld + first);
    }
    // to: the wavefront's share of the stage (a multiple of its size) ^ 1024 turn; the j-th load is of piece j ^ turn
    __device__ __forceinline__ void piece(int j, uint32_t to) const { load_to_lds(base, v[j], to ^ 1024u * j); }
};
// ... and of its reads: operands of sixteen rows (or columns) a step, of half `step` of a stage
template <bool ALONG, int SIDE>
struct TileReads {
    static constexpr int TILES = SIDE / 32;
    uint32_t at[ALONG ? 2 : TILES];
    __device__ __forceinline__ TileReads(int first, int lane) {
        if constexpr (ALONG) {
            const int row = first + (lane & 15);
#pragma unroll
            for (int step = 0; step < 2; ++step) at[step] = (uint32_t)(row * 128 + (((4 * step + (lane >> 4)) ^ pair_mix(row)) << 4));
        } else {
            const int k = 8 * (lane >> 4) + ((lane >> 2) & 3);
#pragma unroll
            for (int i = 0; i < TILES; ++i) at[i] = (uint32_t)(k * SIDE * 2 + (((first / 16 + i) ^ across_swizzle(k)) << 5) + (lane & 3) * 8);
        }
    }
    // half h of operand i; along, the first is all of it
    template <int STEP>
    __device__ __forceinline__ void half(uint32_t stage, int i, int h, bf16x8& whole, shortx4 (&part)[2]) const {
        if constexpr (ALONG) {
            if (h == 0) whole = *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>((uintptr_t)(stage + at[STEP] + 2048u * i));
        } else {
            part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(uintptr_t)(stage + at[i] + 64u * SIDE * STEP + 8u * SIDE * h));
            if (h == 1) whole = __builtin_bit_cast(bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// Units are (tile, range of the contraction), range by range.  XCD x takes a contiguous share of them, its workgroups in turn, so that what runs there at a time
// reads the same operands.
struct Unit { int m0, n0, split, kb, ke; };      // (range in pairs of steps)
template <int SIDE>
struct Units {
    int m_rows, gm, gn, ntiles, k_all, splits, next, end, each;
    __device__ __forceinline__ Units(const VocabProduct& p) {
        m_rows = p.m_count ? *p.m_count : p.m;
        k_all = ((p.k_count ? *p.k_count : p.k) + L_PAIR - 1) / L_PAIR;
        gm = (m_rows + SIDE - 1) / SIDE;
        gn = (p.n + SIDE - 1) / SIDE;
        ntiles = gm * gn;
        splits = p.splits;
        const int units = ntiles * splits, Q = (units + 7) >> 3;
        next = (blockIdx.x & 7) * Q + (blockIdx.x >> 3);
        end = min(((int)(blockIdx.x & 7) + 1) * Q, units);
        each = gridDim.x >> 3;
    }
    __device__ __forceinline__ Unit decode(int u) const {
        const int split = u / ntiles;
        int mi, ni;
        tile_coords(u - split * ntiles, gm, gn, mi, ni);
        auto uniform = [](int x) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(x); };
        return Unit{uniform(mi * SIDE), uniform(ni * SIDE), uniform(split), uniform((int)((int64_t)split * k_all / splits)), uniform((int)((int64_t)(split + 1) * k_all / splits))};
    }
};

template <int SIDE, bool A_ALONG, bool B_ALONG, Epilogue E>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SIDE == 256 ? 1 : 2, SIDE == 256 ? 1 : 2)))
void k_vocab_tile(const VocabProduct p, const typename EpilogueArgs<E>::type e) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int N = SIDE / 32, PIECES = N, STAGE = l_stage(SIDE);      // products a wavefront and side; pieces of its loads of a stage
    constexpr int BEHIND = stores_behind(E, N * N);
    const int wm = (wave >> 1) * (SIDE / 2), wn = (wave & 1) * (SIDE / 2);
    const Units<SIDE> units(p);
    const int m_rows = units.m_rows, k_all = units.k_all, end = units.end, each = units.each;
    int unit = units.next;
    if (unit >= end) return;
    auto decode = [&](int u) __attribute__((always_inline)) { return units.decode(u); };
    floatx4 acc[N][N];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) clear_sum(acc[i][j]);
    };
    auto hold = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) hold_sum(acc[i][j]);
    };
    if (k_all == 0) {                     // a batch without labels
        clear();
        for (; unit < end; unit += each) {
            const Unit x = decode(unit);
            finish(e, p, acc, x.m0 + wm, x.n0 + wn, x.split, lane, m_rows);
        }
        return;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

    // Workgroups that share rows of an operand begin with different pieces of them, so that each meets what another has fetched already.  Loss and gradients of 8192 tokens,
    // width 1280, vocabulary 50257: 4.21 -> 3.9 ms; of 768 tokens, width 768, where three share what they read from memory: 366 -> 378 us.
    auto turn = [&](int first) __attribute__((always_inline)) { return first / SIDE & (PIECES - 1); };
    // The loads run two pairs ahead of the products, into the next unit where the present one ends, so that only the first has to wait for them
    TileLoads<A_ALONG, SIDE> la;
    TileLoads<B_ALONG, SIDE> lb;
    // An operand that is read across ends inside its last pair only where it is the caller's own embedding: rows past its end are its last
    const int tail = B_ALONG ? L_PAIR : p.b.rows - (k_all - 1) * L_PAIR;
    Unit ahead;
    int ahead_unit = unit, at_t;
    bool enter = true;
    auto aim = [&]() __attribute__((always_inline)) {
        if (enter) {
            ahead = decode(ahead_unit);
            la.aim_rows(p.a, ahead.m0, wave, lane, L_PAIR, turn(ahead.n0));
            lb.aim_rows(p.b, ahead.n0, wave, lane, L_PAIR, turn(ahead.m0));
            at_t = ahead.kb;
        }
        if (!B_ALONG && at_t == k_all - 1 && tail < L_PAIR) lb.aim_rows(p.b, ahead.n0, wave, lane, tail, turn(ahead.m0));
        la.aim_pair(p.a, ahead.m0, at_t);
        lb.aim_pair(p.b, ahead.n0, at_t);
        enter = false;
        if (at_t + 1 < ahead.ke) {
            ++at_t;
        } else if (ahead_unit + each < end) {
            ahead_unit += each;
            enter = true;
        }                                 // (behind the last pair of all: that again, for nobody)
    };
    const uint32_t mine = 1024u * PIECES * wave;
    auto next = [&](uint32_t stage) __attribute__((always_inline)) { return stage == (L_STAGES - 1) * STAGE ? 0u : stage + STAGE; };
    const TileReads<A_ALONG, SIDE> ra(wm, lane);
    const TileReads<B_ALONG, SIDE> rb(wn, lane);
    bf16x8 a[2][N], b[2][N];
    // products from register set SET; half 1 - SET of the stages sa, sb goes to the other set, a stage's loads to `to`.  (The products by hand: the compiler would keep
    // some of the sums outside the accumulation registers and spill.  It does not know them for what they are, and would not keep a vector instruction that writes an operand or a sum two wait
    // states away: operands come from LDS; sums that are not fresh come from memory, from the products before, or are zeros, which are held and settled.  The epilogues leave the sums as they are for the same reason.)
    auto step = [&](auto set, auto fresh, uint32_t sa, uint32_t sb, uint32_t to) __attribute__((always_inline)) {
        constexpr int P = decltype(set)::value;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            shortx4 pa[2], pb[2];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if constexpr (decltype(fresh)::value) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=a"(acc[i][j]) : "v"(b[P][j]), "v"(a[P][i]));
                else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[i][j]) : "v"(b[P][j]), "v"(a[P][i]));
                if (j == 0) rb.template half<1 - P>(sb, i, 0, b[P ^ 1][i], pb);
                if (j == 1) rb.template half<1 - P>(sb, i, 1, b[P ^ 1][i], pb);
                if (j == N / 2 - 1) ra.template half<1 - P>(sa, i, 0, a[P ^ 1][i], pa);
                if (j == N / 2) ra.template half<1 - P>(sa, i, 1, a[P ^ 1][i], pa);
                if (j == N - 2) {
                    if constexpr (P == 0) la.piece(i, to);
                    else lb.piece(i, to);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    uint32_t sa = lds0, sb = lds0 + STAGE, to = lds0 + mine;      // of the present pair; of the loads
    for (int d = 0; d < 2; ++d) {
        aim();
#pragma unroll
        for (int j = 0; j < N; ++j) la.piece(j, to ^ 1024 * turn(ahead.n0));
        to += STAGE;
#pragma unroll
        for (int j = 0; j < N; ++j) lb.piece(j, to ^ 1024 * turn(ahead.m0));
        to += STAGE;
    }
    wait_loads<2 * PIECES>();
    lds_barrier();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        shortx4 pa[2], pb[2];
        rb.template half<0>(sb, i, 0, b[0][i], pb);
        rb.template half<0>(sb, i, 1, b[0][i], pb);
        ra.template half<0>(sa, i, 0, a[0][i], pa);
        ra.template half<0>(sa, i, 1, a[0][i], pa);
    }
    uint32_t at = 4 * STAGE, na = 2 * STAGE, nb = 3 * STAGE;  // stage that is loaded next, and those of the next pair
    auto first = [&](auto fresh) __attribute__((always_inline)) {
        aim();
        step(std::integral_constant<int, 0>{}, fresh, sa, sb, (lds0 + at + mine) ^ 1024 * turn(ahead.n0));
        at = next(at);
    };
    auto second = [&]() __attribute__((always_inline)) {
        sa = lds0 + na;
        sb = lds0 + nb;
        step(std::integral_constant<int, 1>{}, std::false_type{}, sa, sb, (lds0 + at + mine) ^ 1024 * turn(ahead.m0));
        at = next(at);
        na = next(nb);
        nb = next(na);
    };
    bool stored = false;
    for (; unit < end; unit += each) {
        const Unit x = decode(unit);
        const int pairs = x.ke - x.kb;
        if constexpr (E == SUMS) {
            clear();
            hold();
            settle();
            begin(e, acc, x.m0 + wm, x.n0 + wn, x.split, lane);
            first(std::false_type{});
        } else {
            first(std::true_type{});
        }
        // The next pair is in LDS, and everyone has read this one.  Behind its loads only the stage above may be on its way; behind a unit also the stores of
        // its results, which were issued after them.
        if (BEHIND > 0 && stored) wait_loads<PIECES + BEHIND>();
        else wait_loads<PIECES>();
        stored = true;
        lds_barrier();
        second();
#pragma unroll 1
        for (int d = 1; d < pairs; ++d) {
            first(std::false_type{});
            wait_loads<PIECES>();
            lds_barrier();
            second();
        }
        // the last product is 18 wait states from its result
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        hold();
        finish(e, p, acc, x.m0 + wm, x.n0 + wn, x.split, lane, m_rows);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                // nothing may arrive in LDS that is not ours any more
}

// ---- the same tiles for numbers of three parts: six products of each step of 32 indices
// The parts of a step are in LDS once, 16 KB each (8), and a part stays in registers for the products that follow one another with it: seven reads of operands instead of
// twelve, and half of the bytes from memory that six separate products would take, which bound them (1378 tokens, width 648, vocabulary 32003, forward and gradients: 1.64 ms, this way 1.35).
// Now, of 343 GFLOP each: statistics 304 us, dz 390, dh 322, dE (by small tiles) 349; matrix instructions are busy in 83 % of the clocks (dz 63).
//   product   a2 b0   a1 b0   a0 b0   a0 b2   a0 b1   a1 b1        register set of a, of b:  0 Q   1 Q   0 Q   0 1-Q   0 Q   1 Q
//   reads     a1      a0      b2      b1      a1      b0, a2 of the next step
//   loads     b0      a2      a1      a0      b2      b1  of the next step
// Ten stages: a part is loaded six products before the one that has its number in this order, and waited for every other product.
constexpr int Q_STAGES = 10;
constexpr int q_stage(int side) { return side * VK * 2; }

template <bool ALONG, int SIDE>
struct PartLoads {
    static constexpr int PIECES = SIDE / 64;        // of 1 KB, a wavefront's of a stage
    uint32_t v[PIECES];
    const char* base;                    // of part 0 of the step
    __device__ __forceinline__ void aim_rows(const VocabOperand& o, int first, int wave, int lane, int turn) {
        const uint32_t row_bytes = 2u * (uint32_t)o.ld;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int piece = PIECES * wave + (j ^ turn);
            if constexpr (ALONG) {
                const int rho = lane >> 2, row = 16 * piece + (((rho & 3) << 2) | (rho >> 2)), u = ((lane & 3) ^ (rho >> 2)) & 3;
                v[j] = (uint32_t)min(row, o.rows - 1 - first) * row_bytes + 16u * u;
            } else {
                constexpr int WORDS = SIDE / 8;      // of 16 bytes, of a contraction index
                const int k = 64 / WORDS * piece + lane / WORDS, col = 16 * ((lane % WORDS >> 1) ^ across_swizzle(k)) + 8 * (lane & 1);
                v[j] = (uint32_t)k * row_bytes + 2u * (uint32_t)min((int64_t)col, o.ld - 8 - first);
            }
        }
    }
    __device__ __forceinline__ void aim_step(const VocabOperand& o, int first, int t) {
        base = reinterpret_cast<const char*>(ALONG ? o.p + (int64_t)first * o.ld + t * VK : o.p + (int64_t)t * VK * o.ld + first);
    }
    // to: the wavefront's share of the stage ^ 1024 turn
    __device__ __forceinline__ void piece(int j, int64_t part_bytes, uint32_t to) const { load_to_lds(base + part_bytes, v[j], to ^ 1024u * j); }
};
template <bool ALONG, int SIDE>
struct PartReads {
    static constexpr int TILES = SIDE / 32;         // of sixteen rows (or columns), a wavefront's
    uint32_t at[ALONG ? 1 : TILES];
    __device__ __forceinline__ PartReads(int first, int lane) {
        if constexpr (ALONG) {
            at[0] = along_unit(first + (lane & 15), lane >> 4);
        } else {
            const int k = 8 * (lane >> 4) + ((lane >> 2) & 3);
#pragma unroll
            for (int i = 0; i < TILES; ++i) at[i] = (uint32_t)(k * SIDE * 2 + (((first / 16 + i) ^ across_swizzle(k)) << 5) + (lane & 3) * 8);
        }
    }
    __device__ __forceinline__ void half(uint32_t stage, int i, int h, bf16x8& whole, shortx4 (&part)[2]) const {
        if constexpr (ALONG) {
            if (h == 0) whole = *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>((uintptr_t)(stage + at[0] + 1024u * i));
        } else {
            part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(uintptr_t)(stage + at[i] + 8u * SIDE * h));
            if (h == 1) whole = __builtin_bit_cast(bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

template <int SIDE, bool A_ALONG, bool B_ALONG, Epilogue E>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SIDE == 256 ? 1 : 2, SIDE == 256 ? 1 : 2)))
void k_vocab_parts_tile(const VocabProduct p, const typename EpilogueArgs<E>::type e) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int N = SIDE / 32, PIECES = SIDE / 64, STAGE = q_stage(SIDE);         // products a wavefront and side; pieces of its loads of a part
    constexpr int BEHIND = stores_behind(E, N * N);
    const int wm = (wave >> 1) * (SIDE / 2), wn = (wave & 1) * (SIDE / 2);
    const Units<SIDE> units(p);
    const int m_rows = units.m_rows, end = units.end, each = units.each;
    int unit = units.next;
    if (unit >= end) return;
    // Small tiles have room to sum the five products of smaller parts for themselves: every one added to the sum of a0 b0 rounds it once more.
    constexpr bool APART = SIDE != VT;
    std::conditional_t<APART, TwoSums, floatx4> acc[N][N];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) clear_sum(acc[i][j]);
    };
    auto hold = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) hold_sum(acc[i][j]);
    };
    if (units.k_all == 0) {               // a batch without labels
        clear();
        for (; unit < end; unit += each) {
            const Unit x = units.decode(unit);
            finish(e, p, acc, x.m0 + wm, x.n0 + wn, x.split, lane, m_rows);
        }
        return;
    }
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

    // The loads run a step ahead of the products, into the next unit where the present one ends.  (Every operand is in the workspace, padded to whole pairs of steps.)
    PartLoads<A_ALONG, SIDE> la;
    PartLoads<B_ALONG, SIDE> lb;
    Unit ahead;
    int ahead_unit = unit, at_t;
    bool enter = true;
    auto turn = [&](int first) __attribute__((always_inline)) { return first / SIDE & (PIECES - 1); };
    auto aim = [&]() __attribute__((always_inline)) {
        if (enter) {
            ahead = units.decode(ahead_unit);
            la.aim_rows(p.a, ahead.m0, wave, lane, turn(ahead.n0));
            lb.aim_rows(p.b, ahead.n0, wave, lane, turn(ahead.m0));
            at_t = 2 * ahead.kb;
        }
        la.aim_step(p.a, ahead.m0, at_t);
        lb.aim_step(p.b, ahead.n0, at_t);
        enter = false;
        if (at_t + 1 < 2 * ahead.ke) {
            ++at_t;
        } else if (ahead_unit + each < end) {
            ahead_unit += each;
            enter = true;
        }                                 // (behind the last step of all: that again, for nobody)
    };
    const int64_t plane_a = 2 * p.a.plane, plane_b = 2 * p.b.plane;
    const uint32_t mine = 1024u * PIECES * wave;
    int base = 0;                                                   // stage of the present step's first part
    auto stage = [&](int n) __attribute__((always_inline)) {        // of part n from there on
        const int x = base + n;
        return lds0 + (uint32_t)(x >= Q_STAGES ? x - Q_STAGES : x) * STAGE;
    };
    // where the wavefront's loads of part n (of the next step: n + 6) go
    auto to_a = [&](int n) __attribute__((always_inline)) { return (stage(n) + mine) ^ 1024 * turn(ahead.n0); };
    auto to_b = [&](int n) __attribute__((always_inline)) { return (stage(n) + mine) ^ 1024 * turn(ahead.m0); };
    const PartReads<A_ALONG, SIDE> ra(wm, lane);
    const PartReads<B_ALONG, SIDE> rb(wn, lane);
    bf16x8 a[2][N], b[2][N];
    // products of sets AS and BS; what stage sa (sb) holds goes to set RA (RB; -1: nothing is read), part `part` of an operand to `to`
    auto product = [&](auto main, auto as, auto bs, auto fresh, auto ra_set, uint32_t sa, auto rb_set, uint32_t sb, auto of_a, int part, uint32_t to) __attribute__((always_inline)) {
        constexpr int AS = decltype(as)::value, BS = decltype(bs)::value, RA = decltype(ra_set)::value, RB = decltype(rb_set)::value;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            shortx4 pa[2], pb[2];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                floatx4* sum;
                if constexpr (!APART) sum = &acc[i][j];
                else if constexpr (decltype(main)::value) sum = &acc[i][j].main;
                else sum = &acc[i][j].low;
                if constexpr (decltype(fresh)::value) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=a"(*sum) : "v"(b[BS][j]), "v"(a[AS][i]));
                else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(*sum) : "v"(b[BS][j]), "v"(a[AS][i]));
                if constexpr (RB >= 0) {
                    if (j == 0) rb.half(sb, i, 0, b[RB][i], pb);
                    if (j == 1) rb.half(sb, i, 1, b[RB][i], pb);
                }
                if constexpr (RA >= 0) {
                    if (j == N / 2 - 1) ra.half(sa, i, 0, a[RA][i], pa);
                    if (j == N / 2) ra.half(sa, i, 1, a[RA][i], pa);
                }
                if (j == N - 2 && (i & 1)) {
                    if constexpr (decltype(of_a)::value) la.piece(i >> 1, part * plane_a, to);
                    else lb.piece(i >> 1, part * plane_b, to);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    constexpr std::integral_constant<int, -1> none;
    constexpr std::integral_constant<int, 0> zero;
    constexpr std::integral_constant<int, 1> one;
    constexpr std::true_type yes;
    constexpr std::false_type no;
    auto meet = [&](bool stored) __attribute__((always_inline)) {   // the parts of this product and the next are in LDS, and everyone is done with the last two
        if (BEHIND > 0 && stored) wait_loads<2 * PIECES + BEHIND>();
        else wait_loads<2 * PIECES>();
        lds_barrier();
    };
    // first: of a unit; fresh: and its sums begin at 0
    auto step = [&](auto q, auto first, auto fresh, bool stored) __attribute__((always_inline)) {
        constexpr std::integral_constant<int, decltype(q)::value> Q;
        constexpr std::integral_constant<int, 1 - decltype(q)::value> R;
        meet(stored);
        aim();
        constexpr std::bool_constant<APART ? decltype(first)::value : decltype(fresh)::value> fresh_first;
        constexpr std::bool_constant<APART && decltype(fresh)::value> fresh_main;
        product(no, zero, Q, fresh_first, one, stage(2), none, 0, no, 0, to_b(6));
        product(no, one, Q, no, zero, stage(3), none, 0, yes, 2, to_a(7));
        meet(false);
        product(yes, zero, Q, fresh_main, none, 0, R, stage(4), yes, 1, to_a(8));
        product(no, zero, R, no, none, 0, Q, stage(5), yes, 0, to_a(9));
        meet(false);
        product(no, zero, Q, no, one, stage(2), none, 0, no, 2, to_b(10));
        const uint32_t load = to_b(11);
        base = base + 6 >= Q_STAGES ? base + 6 - Q_STAGES : base + 6;
        product(no, one, Q, no, zero, stage(1), R, stage(0), no, 1, load);
    };

    aim();
#pragma unroll
    for (int j = 0; j < PIECES; ++j) lb.piece(j, 0, to_b(0));
#pragma unroll
    for (int j = 0; j < PIECES; ++j) la.piece(j, 2 * plane_a, to_a(1));
#pragma unroll
    for (int j = 0; j < PIECES; ++j) la.piece(j, plane_a, to_a(2));
#pragma unroll
    for (int j = 0; j < PIECES; ++j) la.piece(j, 0, to_a(3));
#pragma unroll
    for (int j = 0; j < PIECES; ++j) lb.piece(j, 2 * plane_b, to_b(4));
#pragma unroll
    for (int j = 0; j < PIECES; ++j) lb.piece(j, plane_b, to_b(5));
    wait_loads<4 * PIECES>();
    lds_barrier();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        shortx4 pa[2], pb[2];
        rb.half(stage(0), i, 0, b[0][i], pb);
        rb.half(stage(0), i, 1, b[0][i], pb);
        ra.half(stage(1), i, 0, a[0][i], pa);
        ra.half(stage(1), i, 1, a[0][i], pa);
    }
    bool stored = false;
    for (; unit < end; unit += each) {
        const Unit x = units.decode(unit);
        const int pairs = x.ke - x.kb;
        if constexpr (E == SUMS) {
            clear();
            hold();
            settle();
            begin(e, acc, x.m0 + wm, x.n0 + wn, x.split, lane);
            step(zero, yes, no, stored);
        } else {
            step(zero, yes, yes, stored);
        }
        stored = true;
        step(one, no, no, false);
#pragma unroll 1
        for (int d = 1; d < pairs; ++d) {
            step(zero, no, no, false);
            step(one, no, no, false);
        }
        // the last product is 18 wait states from its result
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        hold();
        finish(e, p, acc, x.m0 + wm, x.n0 + wn, x.split, lane, m_rows);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                // nothing may arrive in LDS that is not ours any more
}

// ---- few tokens: the embedding is read once by each product, straight into registers, and that bounds them
// Operands come as the products want them, 16 bytes of a row to a lane; which four (or eight) contraction indices a lane has is free as long as both operands agree.  Logits of bfloat16 numbers
// on the bfloat16 instructions, everything else in fp32 on its own (16 x 16 x 4): dz is not rounded, and nothing is split into parts.
// A lane has row (column) l % 16 and the indices of l / 16.
// Vocabulary 50257, width 768: of 8 bfloat16 tokens logits take 21 us (77 MB, 3.7 TB/s), of 8 in fp32 39 (154 MB, 4.0 TB/s), dh 26 (5.9 TB/s), dE 32 (4.8); of 40 in fp32 87, 57 and 71: there the
// hidden states (and dz) come from the caches three times as often as the embedding, and bound it.  Handing them round in LDS was slower (four tiles: 155 where these take 104), and so were loads of the
// next tokens under the present products of dE (96 where these take 72: half the wavefronts).
__device__ __forceinline__ void four(const bf16* p, bool there, float (&x)[4]) {
    uint2 w = make_uint2(0, 0);
    if (there) w = *reinterpret_cast<const uint2*>(p);
    x[0] = __uint_as_float(w.x << 16), x[1] = __uint_as_float(w.x & 0xFFFF0000u), x[2] = __uint_as_float(w.y << 16), x[3] = __uint_as_float(w.y & 0xFFFF0000u);
}
__device__ __forceinline__ void four(const float* p, bool there, float (&x)[4]) {
    float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
    if (there) w = *reinterpret_cast<const float4*>(p);
    x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w;
}
template <typename T>
__device__ __forceinline__ floatx4 few_terms(uint4 a, uint4 b, floatx4 c) {
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
    }
}

// Logits: a wavefront takes sixteen rows of the embedding and all tokens, 16 TT at most.  GRAD: dz from them, else their statistics and each label's logit.
struct FewArgs {
    const int* labels;
    float2* stats;                       // [VOCAB_FEW_COLUMNS columns][tokens]
    float* at_label;
    const float *lse, *dloss;
    float* dz;                           // [tokens][few_pitch(vocab)]
};
template <typename T, int TT, bool GRAD>
__global__ __launch_bounds__(256) void k_vocab_few(const T* __restrict__ h, const T* __restrict__ E, int tokens, int W, int V, const FewArgs args) {
    __shared__ float2 part[4][16 * TT];
    constexpr int WORD = 16 / sizeof(T), STEP = 4 * WORD, U = 2;    // numbers of a lane and of a step; steps whose loads are on the way while as many are worked on (eight: 295, not 280 us
    // for 33 fp32 tokens of width 768, vocabulary 50257, with gradients; 63, not 51, for 24 of width 1000, vocabulary 1200: fewer wavefronts a SIMD, and hidden states that leave the first cache)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
    const int v0 = blockIdx.x * VOCAB_FEW_COLUMNS + 16 * wave;
    const T* const e = E + (int64_t)min(v0 + r, V - 1) * W + WORD * g;
    const T* x[TT];
#pragma unroll
    for (int i = 0; i < TT; ++i) x[i] = h + (int64_t)min(16 * i + r, tokens - 1) * W + WORD * g;
    floatx4 acc[TT];
#pragma unroll
    for (int i = 0; i < TT; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    uint4 raw[2][U];
    const int batches = W / (STEP * U);
    auto load = [&](uint4 (&to)[U], int batch) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) to[u] = *reinterpret_cast<const uint4*>(e + STEP * (batch * U + u));
    };
    auto work = [&](const uint4 (&from)[U], int batch) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < TT; ++i) acc[i] = few_terms<T>(from[u], *reinterpret_cast<const uint4*>(x[i] + STEP * (batch * U + u)), acc[i]);
    };
    if (batches > 0) load(raw[0], 0);
    int batch = 0;
    for (; batch + 2 <= batches; batch += 2) {
        load(raw[1], batch + 1);
        work(raw[0], batch);
        if (batch + 2 < batches) load(raw[0], batch + 2);
        work(raw[1], batch + 1);
    }
    if (batch < batches) work(raw[0], batch);
    for (int k = STEP * U * batches; k < W; k += STEP) {            // (a last step may be short: W is a multiple of eight)
        const bool there = k + WORD * g < W;
        const uint4 none = make_uint4(0, 0, 0, 0), b = there ? *reinterpret_cast<const uint4*>(e + k) : none;
#pragma unroll
        for (int i = 0; i < TT; ++i) acc[i] = few_terms<T>(b, there ? *reinterpret_cast<const uint4*>(x[i] + k) : none, acc[i]);
    }
    // acc[i][v]: column v0 + 4 g + v, token 16 i + r
    if constexpr (GRAD) {
#pragma unroll
        for (int i = 0; i < TT; ++i) {
            const int token = 16 * i + r;
            if (token >= tokens) continue;
            const int label = args.labels[token];
            const bool has = label >= 0 && label < V;
            const float lse = args.lse[token], d = args.dloss[token], base = lse * LOG2E;
            // (what that product's rounding loses is made up for as in the tiles)
            const float weight = d * (lse < INFINITY ? exp2_fast(-fmaf(lse, LOG2E, -base)) : 1.f);
            float z[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int col = v0 + 4 * g + v;
                z[v] = has && col < V ? col == label ? d * expm1f(acc[i][v] - lse) : weight * exp2_fast(fmaf(acc[i][v], LOG2E, -base)) : 0.f;
            }
            *reinterpret_cast<float4*>(args.dz + (int64_t)token * few_pitch(V) + v0 + 4 * g) = make_float4(z[0], z[1], z[2], z[3]);
        }
    } else {
        auto larger = [](float a, float b) { return fmaxf(a, b); };
        auto plus = [](float a, float b) { return a + b; };
#pragma unroll
        for (int i = 0; i < TT; ++i) {
            const int token = 16 * i + r, label = token < tokens ? args.labels[token] : -1;
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int col = v0 + 4 * g + v;
                if (col == label && col < V) args.at_label[token] = acc[i][v];
                if (col >= V) acc[i][v] = -INFINITY;
                top = fmaxf(top, acc[i][v]);
            }
            top = apart<32>(apart<16>(top, larger), larger);
            const float base = top == -INFINITY ? 0.f : top * LOG2E;
#pragma unroll
            for (int v = 0; v < 4; ++v) sum += exp2_fast(fmaf(acc[i][v], LOG2E, -base));
            sum = apart<32>(apart<16>(sum, plus), plus);
            if (g == 0) part[wave][16 * i + r] = make_float2(top == -INFINITY ? -INFINITY : base, sum);
        }
        __syncthreads();
        const int mine = threadIdx.x;
        if (mine >= 16 * TT || mine >= tokens) return;
        float2 all = part[0][mine];
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            const float2 o = part[w][mine];
            const float m = fmaxf(all.x, o.x), from = m == -INFINITY ? 0.f : m;
            all = make_float2(m, all.y * exp2_fast(all.x - from) + o.y * exp2_fast(o.x - from));
        }
        args.stats[(int64_t)blockIdx.x * tokens + mine] = all;
    }
}

// dh = dz E: a wavefront takes 64 columns and a range of the vocabulary, sixteen rows of it at a time.  Of a lane's four columns 4 (l % 16) + c each is a product of its
// own, and so is each row 4 (l / 16) + d of the sixteen.
template <typename T, int TT>
__global__ __launch_bounds__(256) void k_vocab_few_dh(const float* __restrict__ dz, const T* __restrict__ E, int tokens, int W, int V, int rows_a_range, float* __restrict__ sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
    const int c0 = blockIdx.y * 256 + 64 * wave + 4 * r;
    const int begin = blockIdx.x * rows_a_range, end = min(begin + rows_a_range, V);
    if ((int)blockIdx.y * 256 + 64 * wave >= W) return;
    const bool there = c0 < W;                                      // (W a multiple of eight)
    const T* const e = E + (there ? c0 : 0);
    const float* z[TT];
#pragma unroll
    for (int i = 0; i < TT; ++i) z[i] = dz + (int64_t)min(16 * i + r, tokens - 1) * few_pitch(V) + 4 * g;
    floatx4 acc[TT][4];
#pragma unroll
    for (int i = 0; i < TT; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[i][c] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
    for (int v = begin; v < end; v += 16) {                         // (dz is 0 behind the vocabulary: its last row stands in for what is missing)
        float y[4][4], x[TT][4];
#pragma unroll
        for (int d = 0; d < 4; ++d) four(e + (int64_t)min(v + 4 * g + d, V - 1) * W, there, y[d]);
#pragma unroll
        for (int i = 0; i < TT; ++i) four(z[i] + v, true, x[i]);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < TT; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[i][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i][d], y[d][c], acc[i][c], 0, 0, 0);
    }
    if (!there) return;
#pragma unroll
    for (int i = 0; i < TT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int token = 16 * i + 4 * g + q;
            if (token < tokens) store4(sums + ((int64_t)blockIdx.x * tokens + token) * W + c0, acc[i][0][q], acc[i][1][q], acc[i][2][q], acc[i][3][q]);
        }
}
// (sixteen shares of the ranges to four numbers: with one, a token's sums are too few to hide behind one another, 17 us for eight tokens)
template <typename T>
__global__ __launch_bounds__(256) void k_vocab_few_sums(const float* __restrict__ sums, const int* __restrict__ labels, int tokens, int W, int V, int ranges, T* __restrict__ dh) {
    __shared__ float4 part[16][16];
    const int q = threadIdx.x & 15, share = threadIdx.x >> 4;
    const int64_t numbers = (int64_t)tokens * W, at = 4 * ((int64_t)blockIdx.x * 16 + q);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float4 y) __attribute__((always_inline)) { x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w); };
    if (at < numbers)
#pragma unroll 8
        for (int i = share; i < ranges; i += 16) add(*reinterpret_cast<const float4*>(sums + i * numbers + at));
    part[share][q] = x;
    __syncthreads();
    if (share || at >= numbers) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) add(part[i][q]);
    const int label = labels[at / W];
    if (label < 0 || label >= V) x = make_float4(0.f, 0.f, 0.f, 0.f);
    store4(dh + at, x.x, x.y, x.z, x.w);
}

// dE = dz^T h: a wavefront takes 64 rows of the vocabulary and 64 columns, sixteen tokens at a time.  Hidden states without a label are not read.
template <typename T>
__global__ __launch_bounds__(256) void k_vocab_few_dE(const float* __restrict__ dz, const T* __restrict__ h, const int* __restrict__ labels, int tokens, int W, int V, T* __restrict__ dE) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
    const int c0 = blockIdx.y * 256 + 64 * wave + 4 * r, v0 = blockIdx.x * 64;
    if ((int)blockIdx.y * 256 + 64 * wave >= W) return;
    const bool there = c0 < W;
    floatx4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[i][c] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int t = 0; t < tokens; t += 16) {
        float y[4][4], x[4][4];
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const int token = t + 4 * g + d, label = token < tokens ? labels[token] : -1;
            four(h + (int64_t)min(token, tokens - 1) * W + (there ? c0 : 0), there && label >= 0 && label < V, y[d]);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i][d] = token < tokens ? dz[(int64_t)token * few_pitch(V) + v0 + 16 * i + r] : 0.f;
        }
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[i][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i][d], y[d][c], acc[i][c], 0, 0, 0);
    }
    if (!there) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int v = v0 + 16 * i + 4 * g + q;
            if (v < V) store4(dE + (int64_t)v * W + c0, acc[i][0][q], acc[i][1][q], acc[i][2][q], acc[i][3][q]);
        }
}

// f(a number of the type, tiles of sixteen tokens)
template <typename F>
void with_few(const mst_vocab_loss_shape& s, F&& f) {
    auto sized = [&](auto type) {
        if (s.tokens <= 16) f(type, std::integral_constant<int, 1>{});
        else f(type, std::integral_constant<int, 2>{});
    };
    if (s.type == MST_BF16) sized(bf16{});
    else if (s.tokens <= 32) sized(float{});
    else if (s.tokens <= 48) f(float{}, std::integral_constant<int, 3>{});
    else f(float{}, std::integral_constant<int, 4>{});
}
static_assert(VOCAB_FEW_BF16 <= 32 && VOCAB_FEW_SMALL <= 32 && VOCAB_FEW_F32 <= 64);

template <bool A_ALONG, bool B_ALONG, Epilogue E>
int launch(const VocabProduct& p, const typename EpilogueArgs<E>::type& e, hipStream_t s) {
    // (as many as the CUs hold: one of 256 x 256, two of 128 x 128)
    auto run = [&](auto kernel, int side, unsigned bytes, uint64_t& done) {
        const unsigned grid = (unsigned)std::min<int64_t>(side == VT ? 256 : 512, 8 * cdiv(cdiv(p.m, side) * cdiv(p.n, side) * p.splits, 8));
        if (int rc = allow_lds(reinterpret_cast<const void*>(kernel), (int)bytes, done)) return rc;
        kernel<<<grid, 256, bytes, s>>>(p, e);
        return (int)MST_OK;
    };
    static uint64_t done[4] = {0, 0, 0, 0};
    int rc = MST_ERR_ARG;
    if constexpr (E != LOGIT_GRAD && E != OUT_BF16) {
        if (p.planes > 1 && p.side == VT) rc = run(k_vocab_parts_tile<VT, A_ALONG, B_ALONG, E>, VT, Q_STAGES * q_stage(VT), done[1]);
        if (p.planes > 1 && p.side != VT) rc = run(k_vocab_parts_tile<VT / 2, A_ALONG, B_ALONG, E>, VT / 2, Q_STAGES * q_stage(VT / 2), done[2]);
    }
    if constexpr (E != LOGIT_GRAD_PARTS && E != OUT_F32) {
        if (p.planes == 1 && p.side == VT) rc = run(k_vocab_tile<VT, A_ALONG, B_ALONG, E>, VT, L_STAGES * l_stage(VT), done[0]);
        if (p.planes == 1 && p.side != VT) rc = run(k_vocab_tile<VT / 2, A_ALONG, B_ALONG, E>, VT / 2, L_STAGES * l_stage(VT / 2), done[3]);
    }
    if (rc) return rc;
    MST_LAUNCH_CHECK();
    return MST_OK;
}

}  // namespace

// Rounds of so many tiles, in rounds of 256 x 256: of 128 x 128 a CU has two at a time, which take 0.62 of the time (twice the loads a product), and one alone 0.4.
static double rounds(int64_t tiles, int side) {
    if (side == VT) return (double)cdiv(tiles, 256);
    const int64_t rest = tiles % 512;
    return 0.62 * (double)(tiles / 512) + (rest == 0 ? 0. : rest <= 256 ? 0.4 : 0.62);
}
// Tiles of 256 x 256 where there are enough of them.  Forward and gradients in us, by the large and by the small ones: bf16 of width 768 and vocabulary 50257, 128 tokens 156 and 127, 600 tokens
// 315 and 288, 1500 tokens 534 and 583; width 1000, vocabulary 1200, 600 tokens 140 and 86 (fp32: 361 and 163); fp32 of width 768 and vocabulary 50257, 128 tokens 560 and 481, 1500 tokens 2392 and 2463.
int vocab_side(int64_t m, int64_t n) {
    return rounds(cdiv(m, VT / 2) * cdiv(n, VT / 2), VT / 2) < rounds(cdiv(m, VT) * cdiv(n, VT), VT) ? VT / 2 : VT;
}
// Tiles, and as many ranges, as let the products end first: each takes as long as its range and what begins and ends it (the time of some eight pairs of steps, the sums of the
// pieces before and behind among it).
void vocab_splits(int m, int n, int k, int& side, int& splits) {
    const int64_t pairs = cdiv(k, L_PAIR);
    double least = 1e30;
    for (int of : {VT, VT / 2})
        for (int s = 1; s <= 64 && s <= pairs; ++s) {
            const double time = rounds(cdiv(m, of) * cdiv(n, of) * s, of) * (double)(cdiv(pairs, s) + 8);
            if (time < least) least = time, side = of, splits = s;
        }
}

int vocab_few(const mst_vocab_loss_shape& s, const void* h, const void* E, const int* labels, float2* stats, float* at_label, hipStream_t stream) {
    with_few(s, [&](auto type, auto tt) {
        using T = decltype(type);
        constexpr int TT = decltype(tt)::value;
        k_vocab_few<T, TT, false><<<(unsigned)cdiv(s.vocab, VOCAB_FEW_COLUMNS), 256, 0, stream>>>(
            static_cast<const T*>(h), static_cast<const T*>(E), s.tokens, s.width, s.vocab, {labels, stats, at_label, nullptr, nullptr, nullptr});
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}
// Ranges of the vocabulary for dh: some thousand workgroups, of 64 rows at least.
int vocab_few_ranges(const mst_vocab_loss_shape& s) {
    return (int)std::min(cdiv(1024, cdiv(s.width, 256)), cdiv(s.vocab, 64));
}
int vocab_few_bwd(const mst_vocab_loss_shape& s, const void* h, const void* E, const int* labels, const float* lse, const float* dloss, float* dz, float* sums, void* dh, void* dE,
                  hipStream_t stream) {
    const int ranges = vocab_few_ranges(s), rows = (int)align_up(cdiv(s.vocab, ranges), 16);
    const unsigned columns = (unsigned)cdiv(s.width, 256);
    with_few(s, [&](auto type, auto tt) {
        using T = decltype(type);
        constexpr int TT = decltype(tt)::value;
        k_vocab_few<T, TT, true><<<(unsigned)cdiv(s.vocab, VOCAB_FEW_COLUMNS), 256, 0, stream>>>(
            static_cast<const T*>(h), static_cast<const T*>(E), s.tokens, s.width, s.vocab, {labels, nullptr, nullptr, lse, dloss, dz});
        if (dh) {
            const int used = (int)cdiv(s.vocab, rows);
            const int64_t numbers = (int64_t)s.tokens * s.width;
            k_vocab_few_dh<T, TT><<<dim3((unsigned)used, columns), 256, 0, stream>>>(dz, static_cast<const T*>(E), s.tokens, s.width, s.vocab, rows, sums);
            k_vocab_few_sums<T><<<(unsigned)cdiv(numbers, 64), 256, 0, stream>>>(sums, labels, s.tokens, s.width, s.vocab, used, static_cast<T*>(dh));
        }
        if (dE)
            k_vocab_few_dE<T><<<dim3((unsigned)cdiv(s.vocab, 64), columns), 256, 0, stream>>>(dz, static_cast<const T*>(h), labels, s.tokens, s.width, s.vocab, static_cast<T*>(dE));
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}

int vocab_stats(const VocabProduct& p, const VocabStats& e, hipStream_t s) { return launch<true, true, STATS>(p, e, s); }
int vocab_logit_grad(const VocabProduct& p, const VocabLogitGrad& e, hipStream_t s) {
    if (p.planes > 1) return launch<true, true, LOGIT_GRAD_PARTS>(p, {e}, s);
    return launch<true, true, LOGIT_GRAD>(p, {e}, s);
}
int vocab_sums(const VocabProduct& p, const VocabSums& e, hipStream_t s) { return launch<true, false, SUMS>(p, e, s); }
int vocab_out(const VocabProduct& p, const VocabOut& e, hipStream_t s) {
    if (e.f32) return launch<false, false, OUT_F32>(p, {e}, s);
    return launch<false, false, OUT_BF16>(p, {e}, s);
}

}  // namespace mst
