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
constexpr int SM = 128, S_OP = SM * 64, S_ROOM = 64 * 128;      // (64 rows of 128 bytes)

enum Epilogue { STATS, LOGIT_GRAD, SUMS, OUT_F32, OUT_BF16 };
template <Epilogue E> struct EpilogueArgs;
template <> struct EpilogueArgs<STATS> { using type = VocabStats; };
template <> struct EpilogueArgs<LOGIT_GRAD> { using type = VocabLogitGrad; };
template <> struct EpilogueArgs<SUMS> { using type = VocabSums; };
template <typename T> struct VocabOutOf : VocabOut {};
template <> struct EpilogueArgs<OUT_F32> { using type = VocabOutOf<float>; };
template <> struct EpilogueArgs<OUT_BF16> { using type = VocabOutOf<bf16>; };

// Results: acc[i][j][v] is row m0 + 16 i + lane % 16, column n0 + 16 j + 4 (lane / 16) + v of C; a wavefront's 16 I rows and 16 J columns.
// A lane's four columns are 8 or 16 bytes of a row; dh and dE go through `room` (the wavefront's own LDS, 16 I rows of ROW bytes) on their way to memory and leave
// it in whole lines.  Word u of row r is kept at u ^ r (of as many as a row has).
template <int ROW>
__device__ __forceinline__ uint32_t room_at(int r, int byte) { return (uint32_t)(r * ROW + ((((byte >> 4) ^ r) & (ROW / 16 - 1)) << 4 | (byte & 15))); }
__device__ __forceinline__ void room_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// f(row, first byte, its word) for the rows r0 .. r0 + ROWS - 1
template <int ROWS, int ROW, typename F>
__device__ __forceinline__ void leave(const char* room, int lane, F&& f) {
    constexpr int EACH = 1024 / ROW;                                // rows of a store
#pragma unroll 8
    for (int r = 0; r < ROWS; r += EACH) {
        const int row = r + lane / (ROW / 16), byte = lane % (ROW / 16) * 16;
        f(row, byte, *reinterpret_cast<const uint4*>(room + room_at<ROW>(row, byte)));
    }
}

// Sums of exp2(z log2 e - base) over 64 columns, those below p.n.  Base is the logit of the row's own label: the sum over all columns is then 1 at least,
// what is lost below fp32 does not count in it, and no maximum has to be found first (a fifth of the instructions).  A sum that leaves fp32 is formed again
// from the row's maximum here.
template <int I, int J, bool ENDS>
__device__ __forceinline__ void statistics(const VocabStats& e, const VocabProduct& p, const floatx4 (&acc)[I][J], int c, int m0, int n0, int lane) {
    const int last = p.n - n0 - 4 * (lane >> 4);
    auto larger = [](float a, float b) { return fmaxf(a, b); };
    auto plus = [](float a, float b) { return a + b; };
    float base[I];
#pragma unroll
    for (int i = 0; i < I; ++i) base[i] = e.at_label[m0 + 16 * i + (lane & 15)] * LOG2E;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        auto z = [&](int j, int v) __attribute__((always_inline)) { return !ENDS || 16 * j + v < last ? acc[i][j][v] : -INFINITY; };
        auto sum_from = [&](float from) __attribute__((always_inline)) {
            float sum = 0.f;
#pragma unroll
            for (int j = c; j < c + 4; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) sum += exp2_fast(fmaf(z(j, v), LOG2E, -from));
            return apart<32>(apart<16>(sum, plus), plus);
        };
        float from = base[i], sum = sum_from(from);
        if (__any(!(sum < INFINITY))) {
            float top = z(c, 0);
#pragma unroll
            for (int j = c; j < c + 4; ++j) top = fmaxf(fmaxf(fmaxf(top, z(j, 0)), fmaxf(z(j, 1), z(j, 2))), z(j, 3));
            from = apart<32>(apart<16>(top, larger), larger) * LOG2E;
            sum = sum_from(from);
        }
        if (lane < 16) e.stats[(int64_t)(e.first + n0 / STAT_COLUMNS + c / 4) * e.row_stride + m0 + 16 * i + lane] = make_float2(from, sum);
    }
}
template <int I, int J>
__device__ __forceinline__ void finish(const VocabStats& e, const VocabProduct& p, floatx4 (&acc)[I][J], int m0, int n0, int, int lane, int, char*) {
#pragma unroll
    for (int c = 0; c < J; c += 4) {
        const int first = n0 + 16 * c;
        if (first + STAT_COLUMNS <= p.n) statistics<I, J, false>(e, p, acc, c, m0, n0, lane);
        else if (first < p.n) statistics<I, J, true>(e, p, acc, c, m0, n0, lane);
    }
}

// dz, straight to memory: a store writes 32 bytes of sixteen rows, and the four that fill a line follow one another.  (Through LDS, in whole lines, it
// waited longer than it saved.)
template <int I, int J, bool ENDS>
__device__ __forceinline__ void logit_grad(const VocabLogitGrad& e, const VocabProduct& p, const floatx4 (&acc)[I][J], int m0, int n0, int lane) {
    const int last = p.n - n0 - 4 * (lane >> 4);
    float base[I], d[I], at_label[I];
    int label[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int m = m0 + 16 * i + (lane & 15);
        base[i] = e.lse[m] * LOG2E;
        d[i] = e.d[m];
        at_label[i] = e.at_label[m];
        label[i] = e.label[m] - e.v0 - n0;
    }
#pragma unroll
    for (int i = 0; i < I; ++i) {
        uint16_t* const row = e.ds + (int64_t)(m0 + 16 * i + (lane & 15)) * e.ld + n0 + 4 * (lane >> 4);
        const bool some = __any(label[i] >= 0 && label[i] < 16 * J);       // of these sixteen rows has its label among these columns (one in 25)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            float x[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] = !ENDS || 16 * j + v < last ? d[i] * exp2_fast(fmaf(acc[i][j][v], LOG2E, -base[i])) : 0.f;
            if (some) {
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (16 * j + 4 * (lane >> 4) + v == label[i]) x[v] = at_label[i];
            }
            uint16_t* to = row + 16 * j;
            for (int part = 0;;) {
                const uint32_t a = pack2(x[0], x[1]), b = pack2(x[2], x[3]);
                *reinterpret_cast<uint2*>(to) = make_uint2(a, b);
                if (++part == p.planes) break;
                to += e.plane;
                x[0] -= __uint_as_float(a << 16);
                x[1] -= __uint_as_float(a & 0xFFFF0000u);
                x[2] -= __uint_as_float(b << 16);
                x[3] -= __uint_as_float(b & 0xFFFF0000u);
            }
        }
    }
}
template <int I, int J>
__device__ __forceinline__ void finish(const VocabLogitGrad& e, const VocabProduct& p, floatx4 (&acc)[I][J], int m0, int n0, int, int lane, int, char*) {
    if (n0 + 16 * J <= p.n) logit_grad<I, J, false>(e, p, acc, m0, n0, lane);
    else logit_grad<I, J, true>(e, p, acc, m0, n0, lane);
}

// fp32 results, half the columns at a time: f(row, column, four results)
template <int I, int J, typename F>
__device__ __forceinline__ void leave_f32(floatx4 (&acc)[I][J], char* room, int lane, F&& f) {
    constexpr int ROW = 32 * J;
#pragma unroll
    for (int c = 0; c < J; c += J / 2) {
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = c; j < c + J / 2; ++j) *reinterpret_cast<floatx4*>(room + room_at<ROW>(16 * i + (lane & 15), 64 * (j - c) + 16 * (lane >> 4))) = acc[i][j];
        room_done();
        leave<16 * I, ROW>(room, lane, [&](int r, int byte, uint4 x) { f(r, 16 * c + byte / 4, __builtin_bit_cast(float4, x)); });
        room_done();
    }
}
// Sums lie as the wavefronts hold them, a wavefront's 16 x 16 results in 1 KB after another (sum_place): the next piece begins with them.
template <int I, int J>
__device__ __forceinline__ float4* sums_of(const VocabSums& e, int m0, int n0, int split, int lane) {
    return reinterpret_cast<float4*>(e.sums + split * e.stride) + sum_place(m0, n0, e.wide) + lane;
}
template <int I, int J>
__device__ __forceinline__ void begin(const VocabSums& e, floatx4 (&acc)[I][J], int m0, int n0, int split, int lane) {
    if (!e.add) return;
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[i][j] = *reinterpret_cast<const floatx4*>(sums_of<I, J>(e, m0 + 16 * i, n0 + 16 * j, split, lane));
}
template <int I, int J, typename Args>
__device__ __forceinline__ void begin(const Args&, floatx4 (&)[I][J], int, int, int, int) {}
template <int I, int J>
__device__ __forceinline__ void finish(const VocabSums& e, const VocabProduct&, floatx4 (&acc)[I][J], int m0, int n0, int split, int lane, int, char*) {
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) *reinterpret_cast<floatx4*>(sums_of<I, J>(e, m0 + 16 * i, n0 + 16 * j, split, lane)) = acc[i][j];
}
template <int I, int J>
__device__ __forceinline__ void finish(const VocabOutOf<float>& e, const VocabProduct& p, floatx4 (&acc)[I][J], int m0, int n0, int, int lane, int m_rows, char* room) {
    const float u = *e.unit;
    leave_f32(acc, room, lane, [&](int r, int c, float4 x) __attribute__((always_inline)) {
        if (m0 + r < m_rows && n0 + c < p.n)
            *reinterpret_cast<float4*>(static_cast<float*>(e.out) + (int64_t)(m0 + r) * e.ld + n0 + c) = make_float4(u * x.x, u * x.y, u * x.z, u * x.w);
    });
}
template <int I, int J>
__device__ __forceinline__ void finish(const VocabOutOf<bf16>& e, const VocabProduct& p, floatx4 (&acc)[I][J], int m0, int n0, int, int lane, int m_rows, char* room) {
    constexpr int ROW = 32 * J;
    const float u = *e.unit;
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j)
            *reinterpret_cast<uint2*>(room + room_at<ROW>(16 * i + (lane & 15), 32 * j + 8 * (lane >> 4))) =
                make_uint2(pack2(u * acc[i][j][0], u * acc[i][j][1]), pack2(u * acc[i][j][2], u * acc[i][j][3]));
    room_done();
    leave<16 * I, ROW>(room, lane, [&](int r, int byte, uint4 x) __attribute__((always_inline)) {
        if (m0 + r < m_rows && n0 + byte / 2 < p.n) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(e.out) + (int64_t)(m0 + r) * e.ld + n0 + byte / 2) = x;
    });
}

template <bool A_ALONG, bool B_ALONG, Epilogue E>
__global__ __launch_bounds__(256) void k_vocab_small(const VocabProduct p, const typename EpilogueArgs<E>::type e) {
    __shared__ __attribute__((aligned(16))) char lds[4 * S_ROOM];        // two operands, then results
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
    begin(e, acc, m0 + wm, n0 + wn, split, lane);
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
    __syncthreads();
    finish(e, p, acc, m0 + wm, n0 + wn, split, lane, m_rows, lds + S_ROOM * wave);
}

// ---- 256 x 256 tiles, four wavefronts of 128 x 128, the sums in the accumulation half of the registers
// A stage of LDS is 64 contraction indices of one operand, 32 KB, so that rows of memory are read in whole lines of 128 bytes; five of them, A and B in turn.
// One wavefront a SIMD has nothing to hide behind: every step's (32 indices') operand reads, for the next step, and a stage's loads, for two to three steps
// after that, stand one by one between its 64 matrix instructions.  Steps come in pairs, of which the second waits for the pair behind it:
//   first   products of its first half, reads of its second half, loads of the next pair but one: A
//   second  waits; products of its second half, reads of the next pair's first half, loads of the next pair but one: B
constexpr int L_PAIR = 2 * VK, L_STAGE = VT * L_PAIR * 2, L_STAGES = 5;
constexpr unsigned L_LDS = L_STAGES * L_STAGE;

// The 16-byte units (eight indices) of a row of an operand along are kept at unit ^ mix(row): sixteen rows of a read cover all banks
__device__ __forceinline__ int pair_mix(int row) { return (row >> 1) & 7; }

// One operand's share of a wavefront's loads: eight pieces of 1 KB a stage
template <bool ALONG>
struct LargeLoads {
    uint32_t v[8];
    const char* base;                    // of the pair
    __device__ __forceinline__ void aim_rows(const VocabOperand& o, int first, int wave, int lane, int left) {
        const uint32_t row_bytes = 2u * (uint32_t)o.ld;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int piece = 8 * wave + j;
            if constexpr (ALONG) {
                const int row = 8 * piece + (lane >> 3), u = (lane & 7) ^ pair_mix(row);
                v[j] = (uint32_t)min(row, o.rows - 1 - first) * row_bytes + 16u * u;
            } else {                     // left: contraction indices from this pair on
                const int k = 2 * piece + (lane >> 5), col = 16 * (((lane & 31) >> 1) ^ across_swizzle(k)) + 8 * (lane & 1);
                v[j] = (uint32_t)min(k, left - 1) * row_bytes + 2u * (uint32_t)min((int64_t)col, o.ld - 8 - first);
            }
        }
    }
    __device__ __forceinline__ void aim_pair(const VocabOperand& o, int first, int part, int t) {
        const uint16_t* const from = o.p + part * o.plane;
        base = reinterpret_cast<const char*>(ALONG ? from + (int64_t)first * o.ld + t * L_PAIR : from + (int64_t)t * L_PAIR * o.ld + first);
    }
    __device__ __forceinline__ void piece(int j, uint32_t to) const { load_to_lds(base, v[j], to + 1024u * j); }
};
// ... and of its reads: eight operands of sixteen rows (or columns) a step, of half `step` of a stage
template <bool ALONG>
struct LargeReads {
    uint32_t at[ALONG ? 2 : 8];
    __device__ __forceinline__ LargeReads(int first, int lane) {
        if constexpr (ALONG) {
            const int row = first + (lane & 15);
#pragma unroll
            for (int step = 0; step < 2; ++step) at[step] = (uint32_t)(row * 128 + (((4 * step + (lane >> 4)) ^ pair_mix(row)) << 4));
        } else {
            const int k = 8 * (lane >> 4) + ((lane >> 2) & 3);
#pragma unroll
            for (int i = 0; i < 8; ++i) at[i] = (uint32_t)(k * 512 + (((first / 16 + i) ^ across_swizzle(k)) << 5) + (lane & 3) * 8);
        }
    }
    // half h of operand i; along, the first is all of it
    template <int STEP>
    __device__ __forceinline__ void half(uint32_t stage, int i, int h, bf16x8& whole, shortx4 (&part)[2]) const {
        if constexpr (ALONG) {
            if (h == 0) whole = *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>((uintptr_t)(stage + at[STEP] + 2048u * i));
        } else {
            part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(uintptr_t)(stage + at[i] + 16384u * STEP + 2048u * h));
            if (h == 1) whole = __builtin_bit_cast(bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

template <bool A_ALONG, bool B_ALONG, Epilogue E>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1)))
void k_vocab_large(const VocabProduct p, const typename EpilogueArgs<E>::type e) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m_rows = p.m_count ? *p.m_count : p.m, k_rows = p.k_count ? *p.k_count : p.k;
    // Workgroup -> (tile, range of the contraction): XCD x takes a contiguous share of them, range by range, so that what runs there at a time
    // reads the same operands
    const int gm = (m_rows + VT - 1) / VT, gn = (p.n + VT - 1) / VT, ntiles = gm * gn, units = ntiles * p.splits, Q = (units + 7) >> 3;
    const int slot = blockIdx.x >> 3, unit = (blockIdx.x & 7) * Q + slot;
    if (slot >= Q || unit >= units) return;
    const int split = unit / ntiles;
    int mi, ni;
    tile_coords(unit - split * ntiles, gm, gn, mi, ni);
    const int m0 = mi * VT, n0 = ni * VT, wm = (wave >> 1) * 128, wn = (wave & 1) * 128;
    const int k_all = (k_rows + L_PAIR - 1) / L_PAIR, per = (k_all + p.splits - 1) / p.splits, kb = min(split * per, k_all), ke = min(kb + per, k_all);
    const int first_term = p.planes == 1 ? 5 : 0, pairs = (ke - kb) * (6 - first_term);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

    LargeLoads<A_ALONG> la;
    LargeLoads<B_ALONG> lb;
    la.aim_rows(p.a, m0, wave, lane, L_PAIR);
    lb.aim_rows(p.b, n0, wave, lane, L_PAIR);
    // An operand that is read across ends inside its last pair only where it is the caller's own embedding (one part): rows past its end are its last
    const int tail = B_ALONG ? L_PAIR : p.b.rows - (k_all - 1) * L_PAIR;
    int at_t = kb, at_term = first_term;  // of the pair that is loaded next; past the end it stays the last
    auto aim = [&]() __attribute__((always_inline)) {
        if (!B_ALONG && at_t == k_all - 1 && tail < L_PAIR) lb.aim_rows(p.b, n0, wave, lane, tail);
        la.aim_pair(p.a, m0, PART_A[at_term], at_t);
        lb.aim_pair(p.b, n0, PART_B[at_term], at_t);
        if (at_t + 1 < ke) ++at_t;
        else if (at_term < 5) ++at_term, at_t = kb;
    };
    const uint32_t mine = 8192u * wave;
    auto next = [&](uint32_t stage) __attribute__((always_inline)) { return stage == (L_STAGES - 1) * L_STAGE ? 0u : stage + L_STAGE; };
    const LargeReads<A_ALONG> ra(wm, lane);
    const LargeReads<B_ALONG> rb(wn, lane);

    floatx4 acc[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    begin(e, acc, m0 + wm, n0 + wn, split, lane);
    bf16x8 a[2][8], b[2][8];
    // products from register set SET; half 1 - SET of the stages sa, sb goes to the other set, a stage's loads to `to`
    auto step = [&](auto set, uint32_t sa, uint32_t sb, uint32_t to) __attribute__((always_inline)) {
        constexpr int P = decltype(set)::value;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            shortx4 pa[2], pb[2];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // (by hand: the compiler would keep some of the sums outside the accumulation registers and spill)
                asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[i][j]) : "v"(b[P][j]), "v"(a[P][i]));
                if (j == 0) rb.template half<1 - P>(sb, i, 0, b[P ^ 1][i], pb);
                if (j == 1) rb.template half<1 - P>(sb, i, 1, b[P ^ 1][i], pb);
                if (j == 3) ra.template half<1 - P>(sa, i, 0, a[P ^ 1][i], pa);
                if (j == 4) ra.template half<1 - P>(sa, i, 1, a[P ^ 1][i], pa);
                if (j == 6) {
                    if constexpr (P == 0) la.piece(i, to);
                    else lb.piece(i, to);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    if (pairs > 0) {
        uint32_t sa = lds0, sb = lds0 + L_STAGE, to = mine;         // (of the present pair; of the loads, from lds0 on)
        for (int d = 0; d < 2; ++d) {
            aim();
#pragma unroll
            for (int j = 0; j < 8; ++j) la.piece(j, lds0 + to);
            to += L_STAGE;
#pragma unroll
            for (int j = 0; j < 8; ++j) lb.piece(j, lds0 + to);
            to += L_STAGE;
        }
        wait_loads<16>();
        lds_barrier();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            shortx4 pa[2], pb[2];
            rb.template half<0>(sb, i, 0, b[0][i], pb);
            rb.template half<0>(sb, i, 1, b[0][i], pb);
            ra.template half<0>(sa, i, 0, a[0][i], pa);
            ra.template half<0>(sa, i, 1, a[0][i], pa);
        }
        uint32_t at = 4 * L_STAGE;                                  // stage that is loaded next, and those of the next pair
        uint32_t na = 2 * L_STAGE, nb = 3 * L_STAGE;
#pragma unroll 1
        for (int d = 0; d < pairs; ++d) {
            aim();
            step(std::integral_constant<int, 0>{}, sa, sb, lds0 + at + mine);
            at = next(at);
            // the next pair is in LDS, and everyone has read this one
            wait_loads<8>();
            lds_barrier();
            sa = lds0 + na;
            sb = lds0 + nb;
            step(std::integral_constant<int, 1>{}, sa, sb, lds0 + at + mine);
            at = next(at);
            na = next(nb);
            nb = next(na);
        }
    }
    // nothing may arrive in LDS that is not ours any more; and the last product is 18 wait states from its result
    asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) asm volatile("" : "+a"(acc[i][j]));
    __syncthreads();
    finish(e, p, acc, m0 + wm, n0 + wn, split, lane, m_rows, lds + 32768 * wave);
}

bool small(int m) { return m <= 128; }

template <bool A_ALONG, bool B_ALONG, Epilogue E>
int launch(const VocabProduct& p, const typename EpilogueArgs<E>::type& e, hipStream_t s) {
    if (small(E == SUMS || E == STATS || E == LOGIT_GRAD ? p.m : p.k)) {
        const int64_t blocks = cdiv(p.m, SM) * cdiv(p.n, SM) * p.splits;
        k_vocab_small<A_ALONG, B_ALONG, E><<<(unsigned)blocks, 256, 0, s>>>(p, e);
    } else {
        static uint64_t done = 0;
        const auto kernel = k_vocab_large<A_ALONG, B_ALONG, E>;
        if (int rc = allow_lds(reinterpret_cast<const void*>(kernel), (int)L_LDS, done)) return rc;
        kernel<<<(unsigned)(8 * cdiv(cdiv(p.m, VT) * cdiv(p.n, VT) * p.splits, 8)), 256, L_LDS, s>>>(p, e);
    }
    MST_LAUNCH_CHECK();
    return MST_OK;
}

}  // namespace

// As many ranges as let the products end first: rounds of 256 workgroups, each as long as its range and what begins and ends it (the time of some eight
// pairs of steps, the sums of the pieces before and behind among it).
int vocab_splits(int m, int n, int k) {
    const int64_t side = small(m) ? SM : VT, tiles = cdiv(m, side) * cdiv(n, side), pairs = cdiv(k, L_PAIR);
    int best = 1;
    int64_t least = INT64_MAX;
    for (int s = 1; s <= 64 && s <= pairs; ++s) {
        const int64_t time = cdiv(tiles * s, 256) * (cdiv(pairs, s) + 8);
        if (time < least) least = time, best = s;
    }
    return best;
}

int vocab_stats(const VocabProduct& p, const VocabStats& e, hipStream_t s) { return launch<true, true, STATS>(p, e, s); }
int vocab_logit_grad(const VocabProduct& p, const VocabLogitGrad& e, hipStream_t s) { return launch<true, true, LOGIT_GRAD>(p, e, s); }
int vocab_sums(const VocabProduct& p, const VocabSums& e, hipStream_t s) { return launch<true, false, SUMS>(p, e, s); }
int vocab_out(const VocabProduct& p, const VocabOut& e, hipStream_t s) {
    if (e.f32) return launch<false, false, OUT_F32>(p, {e}, s);
    return launch<false, false, OUT_BF16>(p, {e}, s);
}

}  // namespace mst
