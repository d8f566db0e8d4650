// Gradients of the attention over selected blocks (mst_block_attention_bwd).  With P = exp(scale q.k - lse),
// delta = sum of dO O over a row and dP = dO V^T:  dS = P (dP - delta),  dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K.
//
// The first kernel walks lists of the queries of each block: a workgroup takes a stretch of the rows that selected a block, whose keys and values its
// wavefronts keep in registers, 32 keys each.  The rows' Q and dO come straight to LDS, each from its own address, and are read
// along the rows for S and dP and across them for dK and dV, whose sums stay in registers: no two workgroups meet in one
// sum.  A block with one item is written as it is; the sums of several items are left in fp32 and added in the order of the list.
// The second works like the forward: rows that own their dQ walk the union of their blocks.
//
// Measured, 8192 queries of 20 heads of 64, 8 blocks of 64: lists 30 us, dK and dV 147 (270 TFLOP/s of the rows' own pairs), their sums 12, delta 19, dQ 216 (the union:
// three and a half times the blocks of a row).  2 x 4099 of 24 heads of 128 with 8 key heads: dK and dV 323 us (one wavefront a SIMD, bound by the time from a
// load to its use; matrix instructions busy in 17 % of the clocks), dQ 218.
// A row's weights are cut into 0 .. 1 and multiplied so that 0 times anything is 0: what a row does not see has no part in its dQ, also where the scores
// or dP of that left fp32.
//
// dQ is a difference: the rows of dS add up to zero, and what the keys have in common falls out.  An error in delta, or one in
// dS that does not add up to zero, brings it back.  delta from the rounded O is off by a bfloat16 rounding of O, and a bfloat16 dS by its own:
// with keys of a common direction dQ was 3.5e-3 off (2-norm; its own rounding makes 1.7e-3).  So the first kernel, which has
// dS with that delta in fp32, also leaves the sum of each of its rows, which is what delta lacks; a small launch adds them; and
// the second takes dS as two bfloat16 numbers, high and low: 1.7e-3.  The first takes dS and P so too: rounded once, they put dK 2.4e-3 to 3.0e-3 off
// and dV 2.4e-3, as two numbers 1.9e-3 and 1.7e-3, for 14 us of 131 (8192 queries of 20 heads of 64; 35 of 288 for 2 x 4099 of 24 of 128).  (What dK still has is delta's error.)
#include "block_rows.h"

namespace mst {
namespace {

constexpr size_t PARTIAL_BYTES = size_t(256) << 20;

// x y, and 0 if either is 0, whatever the other is (one instruction, as an ordinary product)
__device__ float product_or_zero(float x, float y) __asm("llvm.amdgcn.fmul.legacy");

struct BwdArgs {
    const float* lse;                    // [B][H][Tq]
    const float* delta;                  // [B][H][Tq]
    float* dkv;                          // [item][2][BK][D]
    float* lack;                         // [pair][R] sums of rows of dS over a block (bfloat16 operands)
};

template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_attention_delta(AttentionArgs a, Heads<const T> o, Heads<const T> d_o, float* __restrict__ delta) {
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;     // (query, head)
    if (row >= (int64_t)a.Tq * a.H) return;
    const int t = (int)(row / a.H), h = (int)(row - (int64_t)t * a.H), b = blockIdx.y;
    float x[8], y[8], s = 0.f;
    if (lane * 8 < a.D) {
        load8(o.at(b, t, h) + lane * 8, x);
        load8(d_o.at(b, t, h) + lane * 8, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += x[e] * y[e];
    }
    s = lanes_sum<LANES>(s);
    if (lane == 0) delta[((int64_t)b * a.H + h) * a.Tq + t] = s;
}

// a workgroup of dK and dV: KP parts of 32 keys times RG groups of 32 rows, a wavefront each
template <typename T, int DP, int KP>
struct DkvTiles {
    using R = Rows<T, DP>;
    static constexpr int RG = KP == 4 ? 1 : 2, WAVES = KP * RG, THREADS = WAVES * 64, RT = RG * 32;
    static constexpr int TILE = RT * R::BYTES, BUFFER = 2 * TILE, EACH = BUFFER / 1024 / WAVES;      // Q and dO of RT rows
    static constexpr int ROWS = 2 * BUFFER, STATS = ROWS + 2 * 2 * RT * 8, LACK = STATS + 2 * RT * 12, BYTES = LACK + 2 * (KP + 1) * RT * 4;   // LDS: where a row's Q and dO are, its statistics, sums of dS
    static_assert(TILE % (EACH * 1024) == 0 && BUFFER * 2 >= (RG - 1) * KP * 32 * DP * 8, "whole loads; room for the sums of half the wavefronts");
};

// (128 components take more registers than two wavefronts a SIMD have: so bound, it spills 170 bytes a lane, and 4099 queries of 24 heads
// with 8 key heads take 368 us, not 281, P and dS rounded once)
template <typename T, int DP, int KP>
__global__ __launch_bounds__((DkvTiles<T, DP, KP>::THREADS), (sizeof(T) * DP >= 256 ? 1 : 2)) void k_attention_dkv(AttentionArgs a, Lists lists, Heads<const T> q, Heads<const T> k, Heads<const T> v,
                                                                               Heads<const T> d_o, int bg0, int group, BwdArgs w, Heads<T> dk_out, Heads<T> dv_out) {
    using Tiles = DkvTiles<T, DP, KP>;
    using R = Rows<T, DP>;
    constexpr int QC = DP / 16, DT = DP / 32, RT = Tiles::RT, RG = Tiles::RG, EACH = Tiles::EACH;
    extern __shared__ __align__(16) char lds[];
    // the items of a key head lie `group` workgroups apart: mostly on one XCD, whose L2 then holds the head's queries
    const int index = blockIdx.x / group, in_group = blockIdx.x - index * group, bg = bg0 + in_group, b = bg / a.G, g = bg % a.G;
    if (index >= lists.item_start[(int64_t)in_group * (a.nb + 1) + a.nb]) return;
    const int2 it = lists.items[(int64_t)in_group * lists.max_items + index];
    const int block = it.x, first = it.y, end = lists.start[(int64_t)in_group * (a.nb + 1) + block + 1], pairs = min(lists.item_pairs, end - first);
    const bool alone = pairs == end - first && lists.start[(int64_t)in_group * (a.nb + 1) + block] == first;      // the block's only item
    const int len = a.length(b), key0 = block * a.BK;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i32 = lane & 31, half = lane >> 5;
    const int kp = wave % KP, rg = wave / KP, key = key0 + kp * 32 + i32;
    const float scale2 = a.scale * LOG2E, inv_r = 1.f / (float)a.R;

    Operand<T> kf[QC], vf[QC];           // columns = keys
#pragma unroll
    for (int c = 0; c < QC; ++c) {
        const int d = c * 16 + half * 8;
        const bool there = key < len && d < a.D;
        kf[c] = there ? load_operand(k.at(b, key, g) + d) : zero_operand<T>();
        vf[c] = there ? load_operand(v.at(b, key, g) + d) : zero_operand<T>();
    }
    floatx16 dk[DT], dv[DT];             // rows = components, columns = keys
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[d] = dv[d] = zero16();

    // The rows of step x are known two steps ahead (their queries, by the first RT threads) and their statistics one.
    const int rows = pairs * a.R, steps = (rows + RT - 1) / RT;
    const int* list = lists.list + (int64_t)in_group * a.Tq * a.NS + first;
    int64_t* row_at = reinterpret_cast<int64_t*>(lds + Tiles::ROWS);               // [2][2][RT] byte offsets of a row's Q and dO from the batch's
    float* stats = reinterpret_cast<float*>(lds + Tiles::STATS);                   // [2][3][RT] log-sum, delta, last key that it sees
    const bool scout = (int)threadIdx.x < RT;
    const bool is_q = wave < Tiles::WAVES / 2;
    const char* base = reinterpret_cast<const char*>(is_q ? q.at(b, 0, g * a.R) : d_o.at(b, 0, g * a.R));
    const uint32_t to = lds_address(lds) + wave * (EACH * 1024);
    const int my_row = (wave % (Tiles::WAVES / 2)) * EACH * R::PER_KB + lane / R::CH;
    int chunk[EACH];                     // a lane's chunk of a row
#pragma unroll
    for (int i = 0; i < EACH; ++i) chunk[i] = min(((lane % R::CH) ^ R::mix(my_row + i * R::PER_KB)) * 16, a.D * (int)sizeof(T) - 16);
    auto row_of = [&](int x) {           // pair and head of the thread's row of step x; rows past the last are read as that
        const int row = min(x * RT + (int)threadIdx.x, rows - 1);
        const int e = (int)(((float)row + 0.5f) * inv_r);      // (rows are below 2^13, heads up to 64: never within rounding of the next one)
        return make_int2(list[e], row - e * a.R);              // (its pair)
    };
    // where the sum of a row of dS goes: for each buffer the sums of the KP parts and the row's place (-1 behind the rows)
    float* lack = reinterpret_cast<float*>(lds + Tiles::LACK);
    auto put_place = [&](int2 th, int x) {
        const int place = ((th.x >> SELECT_BITS) * a.NS + (th.x & (SELECT_MAX - 1))) * a.R + th.y;
        reinterpret_cast<int*>(lack)[(x & 1) * (KP + 1) * RT + KP * RT + threadIdx.x] = x * RT + (int)threadIdx.x < rows ? place : -1;
    };
    auto store_lack = [&](int x) {
        const float* p = lack + (x & 1) * (KP + 1) * RT + threadIdx.x;
        const int place = __float_as_int(p[KP * RT]);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < KP; ++i) sum += p[i * RT];
        if (place >= 0) w.lack[(int64_t)in_group * a.Tq * a.NS * a.R + place] = sum;
    };
    struct Stat { float lse, delta; int limit; };
    auto stat_of = [&](int2 th, int x) {
        const int t = th.x >> SELECT_BITS;
        const int64_t at = ((int64_t)b * a.H + g * a.R + th.y) * a.Tq + t;
        const float lse = w.lse[at];                           // (-inf: all scores are; weights 2^-inf)
        return Stat{lse == -INFINITY ? INFINITY : lse * LOG2E, w.delta[at], x * RT + (int)threadIdx.x < rows ? len - a.Tq + t - key0 : -1};
    };
    auto put_stat = [&](const Stat& s, int x) {
        float* p = stats + (x & 1) * 3 * RT + threadIdx.x;
        p[0] = s.lse, p[RT] = s.delta, p[2 * RT] = __int_as_float(s.limit);
    };
    auto put_row = [&](int2 th, int x) {
        int64_t* p = row_at + (x & 1) * 2 * RT + threadIdx.x;
        const int t = th.x >> SELECT_BITS;
        p[0] = (t * q.st + th.y * q.sh) * (int64_t)sizeof(T), p[RT] = (t * d_o.st + th.y * d_o.sh) * (int64_t)sizeof(T);
    };
    auto load_rows = [&](int x) {
        const int64_t* row = row_at + ((x & 1) * 2 + (is_q ? 0 : 1)) * RT + my_row;
#pragma unroll
        for (int i = 0; i < EACH; ++i) gather_to_lds(base + (row[i * R::PER_KB] + chunk[i]), to + (x & 1) * Tiles::BUFFER + i * 1024);
    };
    constexpr bool LACKS = sizeof(T) == 2;
    int2 th1 = make_int2(0, 0), th2 = th1;
    Stat stat1{0.f, 0.f, -1};
    if (scout) {
        const int2 th0 = row_of(0);
        th1 = row_of(1);
        th2 = row_of(2);
        if (LACKS) put_place(th0, 0);
        put_row(th0, 0), put_row(th1, 1);
        put_stat(stat_of(th0, 0), 0);
        stat1 = stat_of(th1, 1);
    }
    lds_barrier();
    load_rows(0);
    for (int x = 0; x < steps; ++x) {
        wait_loads<0>();
        lds_barrier();
        const char *qt = lds + (x & 1) * Tiles::BUFFER, *ot = qt + Tiles::TILE;
        if (x + 1 < steps) load_rows(x + 1);
        if (LACKS && scout && x > 0) store_lack(x - 1);
        if (scout && x + 1 < steps) {
            if (LACKS) put_place(th1, x + 1);
            put_stat(stat1, x + 1);
            th1 = th2;
            put_row(th2, x);
            stat1 = stat_of(th2, x + 2);
            th2 = row_of(x + 3);
        }
        floatx16 s = zero16(), dp = zero16();
#pragma unroll
        for (int c = 0; c < QC; ++c) {
            if (!worth<T>(c * 16, a.D)) continue;
            s = product32(along_row<T, DP>(qt, rg * 32 + i32, c * 16 + half * 8), kf[c], s);
            dp = product32(along_row<T, DP>(ot, rg * 32 + i32, c * 16 + half * 8), vf[c], dp);
        }
        const float* stat = stats + (x & 1) * 3 * RT + rg * 32 + 4 * half;
        // rows that see all of this part's keys need no comparison (those of later blocks, which are most)
        const bool cut = __any(__float_as_int(stats[(x & 1) * 3 * RT + 2 * RT + rg * 32 + i32]) < kp * 32 + 31);
        float row_sum[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float p[8], ds[8];
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const float4 ls = *reinterpret_cast<const float4*>(stat + u * 16 + 2 * e), de = *reinterpret_cast<const float4*>(stat + RT + u * 16 + 2 * e);
                const float l4[4] = {ls.x, ls.y, ls.z, ls.w}, d4[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int n = u * 8 + e + r;
                    p[e + r] = exp2_fast(__builtin_fmaf(s[n], scale2, -l4[r]));
                    ds[e + r] = p[e + r] * (dp[n] - d4[r]);
                }
                if (cut) {
                    const int4 li = *reinterpret_cast<const int4*>(stat + 2 * RT + u * 16 + 2 * e);
                    const int i4[4] = {li.x, li.y, li.z, li.w};
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (kp * 32 + i32 > i4[r]) p[e + r] = ds[e + r] = 0.f;
                }
            }
            Operand<T> pf, sf, p_low, s_low;       // columns = keys, contraction over the rows
            set_operand(pf, p);
            set_operand(sf, ds);
            set_operand_rest(p_low, pf, p);
            set_operand_rest(s_low, sf, ds);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                if (!worth<T>(d * 32, a.D)) continue;
                const Operand<T> grads = across_rows<T, DP>(ot, rg * 32 + u * 16, d * 32, lane);
                dv[d] = product32(grads, pf, dv[d]);
                if (sizeof(T) == 2) dv[d] = product32(grads, p_low, dv[d]);
                const Operand<T> queries = across_rows<T, DP>(qt, rg * 32 + u * 16, d * 32, lane);
                dk[d] = product32(queries, sf, dk[d]);
                if (sizeof(T) == 2) dk[d] = product32(queries, s_low, dk[d]);
            }
            if (LACKS)
#pragma unroll
                for (int e = 0; e < 4; ++e) row_sum[u * 4 + e] = sixteen_apart_sum(ds[2 * e], ds[2 * e + 1]);
        }
        if (LACKS) {
            // rows of 16 lanes (half, odd): sums over their lanes of the registers 2j + odd; lane j keeps the jth
            float mine = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float sum = lanes_sum<16>(row_sum[j]);
                if ((lane & 15) == j) mine = sum;
            }
            const int n = 2 * (lane & 7) + ((lane >> 4) & 1);
            if ((lane & 15) < 8) lack[((x & 1) * (KP + 1) + kp) * RT + rg * 32 + 8 * (n / 4) + 4 * half + n % 4] = mine;
        }
    }
    __syncthreads();
    if (LACKS && scout) store_lack(steps - 1);
    if (RG == 2) {                       // the second group of rows to the first
        float* sums = reinterpret_cast<float*>(lds) + kp * (DT * 32 * 64) + lane;
        if (rg == 1)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) sums[(d * 32 + r) * 64] = dk[d][r], sums[(d * 32 + 16 + r) * 64] = dv[d][r];
        __syncthreads();
        if (rg == 1) return;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) dk[d][r] += sums[(d * 32 + r) * 64], dv[d][r] += sums[(d * 32 + 16 + r) * 64];
    }
    if (alone) {
        if (key >= a.S) return;
        T *pk = dk_out.at(b, key, g), *pv = dv_out.at(b, key, g);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int c = d * 32 + 2 * r + 4 * half;
                if (c >= a.D) continue;
                store4(pk + c, dk[d][r] * a.scale, dk[d][r + 1] * a.scale, dk[d][r + 2] * a.scale, dk[d][r + 3] * a.scale);
                store4(pv + c, dv[d][r], dv[d][r + 1], dv[d][r + 2], dv[d][r + 3]);
            }
        return;
    }
    float* out = w.dkv + (((int64_t)in_group * lists.max_items + index) * 2 * a.BK + kp * 32 + i32) * a.D;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int c = d * 32 + 2 * r + 4 * half;
            if (c >= a.D) continue;
            store4(out + c, dk[d][r], dk[d][r + 1], dk[d][r + 2], dk[d][r + 3]);
            store4(out + (int64_t)a.BK * a.D + c, dv[d][r], dv[d][r + 1], dv[d][r + 2], dv[d][r + 3]);
        }
}

// delta of a row and what it lacked, block after block
__global__ __launch_bounds__(256) void k_attention_delta_whole(AttentionArgs a, Plan plan, int bg0, const float* __restrict__ lack, float* __restrict__ delta) {
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;                       // (query, head) of a key head
    if (row >= (int64_t)a.Tq * a.R) return;
    const int t = (int)(row / a.R), h = (int)(row - (int64_t)t * a.R), bg = bg0 + blockIdx.y, b = bg / a.G, g = bg % a.G;
    const int* blocks = plan.rows + ((int64_t)bg * a.Tq + t) * a.NS;
    const float* p = lack + ((int64_t)blockIdx.y * a.Tq + t) * a.NS * a.R + h;
    float sum = 0.f;
    for (int s = 0; s < a.NS && blocks[s] < a.nb; ++s) sum += p[s * a.R];
    delta[((int64_t)b * a.H + g * a.R + h) * a.Tq + t] += sum;
}

// dK and dV of four components of a key whose block has no item or several: their sum, in order
template <typename T>
__global__ __launch_bounds__(256) void k_attention_dkv_join(AttentionArgs a, Lists lists, int bg0, BwdArgs w, Heads<T> dk, Heads<T> dv) {
    const int bg = bg0 + blockIdx.y, b = bg / a.G, g = bg % a.G, units = a.D / 4;
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t key = u / units;
    if (key >= a.S) return;
    const int d = (int)(u - key * units) * 4, block = (int)(key / a.BK), in = (int)(key - (int64_t)block * a.BK);
    const int i0 = lists.item_start[(int64_t)blockIdx.y * (a.nb + 1) + block], i1 = lists.item_start[(int64_t)blockIdx.y * (a.nb + 1) + block + 1];
    if (i1 - i0 == 1) return;
    float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = i0; i < i1; ++i) {
        const float* p = w.dkv + (((int64_t)blockIdx.y * lists.max_items + i) * 2 * a.BK + in) * a.D + d;
        const float4 s = *reinterpret_cast<const float4*>(p), z = *reinterpret_cast<const float4*>(p + (int64_t)a.BK * a.D);
        x[0] += s.x; x[1] += s.y; x[2] += s.z; x[3] += s.w;
        y[0] += z.x; y[1] += z.y; y[2] += z.z; y[3] += z.w;
    }
    store4(dk.at(b, key, g) + d, x[0] * a.scale, x[1] * a.scale, x[2] * a.scale, x[3] * a.scale);
    store4(dv.at(b, key, g) + d, y[0], y[1], y[2], y[3]);
}

// (three workgroups a CU at 64 components of 2 bytes, 168 registers without spilling: 8192 queries of 20 heads 236 -> 215 us, 4 x 1024 of 12
// heads, too few workgroups to fill the card, 32.3 -> 33.2.  More components, or wider ones, take the registers of two or of one.)
template <typename T, int DP, int KW>
__global__ __launch_bounds__(ROW_THREADS, (sizeof(T) * DP == 512 ? 1 : sizeof(T) * DP == 128 ? 3 : 2)) void k_attention_dq(AttentionArgs a, Plan plan, UnionSpace space, int tiles, Heads<const T> q, Heads<const T> k, Heads<const T> v,
                                                                 Heads<const T> d_o, const float* __restrict__ lse, const float* __restrict__ delta, Heads<T> dq) {
    using Tiles = KeyTiles<T, DP, KW>;
    constexpr int QC = DP / 16, DT = DP / 32, ST = KW / 32;
    extern __shared__ __align__(16) char lds[];
    const RowWork work(tiles);
    const int bg = work.bg, b = bg / a.G, g = bg % a.G, len = a.length(b), tokens = COLS / a.R, t0 = work.tile * tokens;
    uint32_t* list = reinterpret_cast<uint32_t*>(lds + space.list);
    uint16_t* rows = reinterpret_cast<uint16_t*>(lds + space.rows);
    const int n = make_union(a, plan.rows + (int64_t)bg * a.Tq * a.NS, t0, tokens, reinterpret_cast<uint32_t*>(lds + space.words), list, rows);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i32 = lane & 31, half = lane >> 5;
    const int col = wave * 32 + i32, tok = col / a.R, t = t0 + tok, h = g * a.R + col - tok * a.R;
    const bool there = tok < tokens && t < a.Tq;
    const int p = len - a.Tq + t;
    const int64_t stat = ((int64_t)b * a.H + (there ? h : 0)) * a.Tq + (there ? t : 0);
    const float lse2 = lse[stat] * LOG2E, dl = delta[stat];
    // a positive factor, so that -inf is below every score: its sign goes to the query
    const float scale2 = fmaxf(fabsf(a.scale) * LOG2E, 1.17549435e-38f);
    Operand<T> qf[QC], of[QC];
    const T *qp = q.at(b, there ? t : 0, there ? h : 0), *op = d_o.at(b, there ? t : 0, there ? h : 0);
#pragma unroll
    for (int c = 0; c < QC; ++c) {
        const int d = c * 16 + half * 8;
        qf[c] = there && d < a.D ? load_operand(qp + d) : zero_operand<T>();
        if (a.scale < 0.f) qf[c] = negated(qf[c]);
        of[c] = there && d < a.D ? load_operand(op + d) : zero_operand<T>();
    }
    floatx16 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = zero16();
    Cursor cursor(a, rows, tok, there);
    const Tiles tiles_in(a, k, v, b, g, wave, lds);
    const int parts = a.BK / KW, all = n * parts;
    auto entry_of = [&](int i) { return (uint32_t)__builtin_amdgcn_readfirstlane(list[i]); };
    uint32_t entry = n > 0 ? entry_of(0) : 0;
    if (n > 0) tiles_in.load((int)(entry & 0xFFFF) * a.BK, len, 0);
    for (int x = 0, i = 0, part = 0; x < all; ++x) {
        wait_loads<0>();
        lds_barrier();
        const uint32_t now = entry;
        const int key0 = (int)(now & 0xFFFF) * a.BK + part * KW;
        const char* tile = lds + (x & 1) * Tiles::BUFFER;
        const bool block_ends = part + 1 == parts;
        if (x + 1 < all) {
            if (block_ends) entry = entry_of(i + 1);
            tiles_in.load(block_ends ? (int)(entry & 0xFFFF) * a.BK : key0 + KW, len, (x + 1) & 1);
        }
        part = block_ends ? 0 : part + 1;
        i += block_ends;
        if ((now >> (16 + wave)) & 1) {
            const int limit = cursor.next == (int)(now & 0xFFFF) ? p - key0 : -1;
            const bool cut = __any(limit < KW - 1 && limit >= 0);          // some row sees some of these keys, not all
            const float less = limit < 0 ? INFINITY : lse2;    // a row that sees nothing here: weights 2^-inf
#pragma unroll
            for (int st = 0; st < ST; ++st) {
                floatx16 s = zero16(), dp = zero16();
#pragma unroll
                for (int c = 0; c < QC; ++c) {
                    s = product32(along_row<T, DP>(tile, st * 32 + i32, c * 16 + half * 8), qf[c], s);
                    dp = product32(along_row<T, DP>(tile + Tiles::TILE, st * 32 + i32, c * 16 + half * 8), of[c], dp);
                }
                if (cut)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (st * 32 + 8 * (r / 4) + 4 * half + r % 4 > limit) s[r] = -INFINITY;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {          // (0 for what a row does not see, also where s or dp left fp32: the median of no number is 0)
                        const float weight = __builtin_amdgcn_fmed3f(exp2_fast(__builtin_fmaf(s[u * 8 + e], scale2, -less)), 0.f, 1.f);
                        y[e] = product_or_zero(weight, dp[u * 8 + e] - dl);
                    }
                    Operand<T> sf, low;
                    set_operand(sf, y);
                    set_operand_rest(low, sf, y);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        if (!worth<T>(d * 32, a.D)) continue;
                        const Operand<T> keys = across_rows<T, DP>(tile, st * 32 + u * 16, d * 32, lane);
                        acc[d] = product32(keys, sf, acc[d]);
                        if (sizeof(T) == 2) acc[d] = product32(keys, low, acc[d]);
                    }
                }
            }
        }
        if (block_ends) cursor.pass(a, (int)(now & 0xFFFF));
    }
    if (!there) return;
    const float scale = lse2 == lse2 ? a.scale : lse2;             // (a row whose scores are no numbers: the weights above were cut to 0)
    T* po = dq.at(b, t, h);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int c = d * 32 + 2 * r + 4 * half;
            if (c < a.D) store4(po + c, acc[d][r] * scale, acc[d][r + 1] * scale, acc[d][r + 2] * scale, acc[d][r + 3] * scale);
        }
}

struct BwdSpace {
    int group;                           // (batch, key head) that a launch takes
    size_t lists, delta, dkv, total;
};

BwdSpace bwd_space(const mst_attention_shape* s) {
    const AttentionArgs a = attention_args(s);
    BwdSpace w;
    const Lists lists = carve_lists(nullptr, a, 1);
    w.delta = align_up((size_t)a.B * a.H * a.Tq * 4);
    const size_t one = (size_t)lists.max_items * 2 * a.BK * a.D * 4, lack = s->type == MST_BF16 ? (size_t)a.Tq * a.NS * a.R * 4 : 0;
    w.group = (int)std::min<size_t>((size_t)a.B * a.G, std::max<size_t>(1, PARTIAL_BYTES / std::max<size_t>(lists.total + one + lack, 1)));
    w.lists = carve_lists(nullptr, a, w.group).total;
    w.dkv = align_up(w.group * one);
    w.total = std::max<size_t>(256, w.lists + w.delta + w.dkv + align_up(w.group * lack));
    return w;
}

template <typename T, int DP, int KP>
int launch_dkv(const AttentionArgs& a, const Plan& plan, const Lists& lists, const BwdSpace& sp, const Heads<const T>& q, const Heads<const T>& k, const Heads<const T>& v, const Heads<const T>& d_o,
               const Heads<T>& dk, const Heads<T>& dv, const BwdArgs& w, hipStream_t st) {
    using Tiles = DkvTiles<T, DP, KP>;
    static_assert(Tiles::BYTES <= LDS_BYTES, "LDS of a CU");
    static uint64_t allowed = 0;
    if (int e = allow_lds(reinterpret_cast<const void*>(&k_attention_dkv<T, DP, KP>), Tiles::BYTES, allowed)) return e;
    for (int bg = 0; bg < a.B * a.G; bg += sp.group) {
        const unsigned n = (unsigned)std::min(sp.group, a.B * a.G - bg);
        if (int e = build_lists(a, plan, lists, bg, (int)n, st)) return e;
        k_attention_dkv<T, DP, KP><<<(unsigned)lists.max_items * n, Tiles::THREADS, Tiles::BYTES, st>>>(a, lists, q, k, v, d_o, bg, (int)n, w, dk, dv);
        MST_LAUNCH_CHECK();
        k_attention_dkv_join<T><<<dim3((unsigned)cdiv((int64_t)a.S * (a.D / 4), 256), n), 256, 0, st>>>(a, lists, bg, w, dk, dv);
        MST_LAUNCH_CHECK();
        if (sizeof(T) == 2 && a.Tq > 0) {
            k_attention_delta_whole<<<dim3((unsigned)cdiv((int64_t)a.Tq * a.R, 256), n), 256, 0, st>>>(a, plan, bg, w.lack, const_cast<float*>(w.delta));
            MST_LAUNCH_CHECK();
        }
    }
    return MST_OK;
}

template <typename T, int DP, int KW>
int launch_dq(const AttentionArgs& a, const Plan& plan, const Heads<const T>& q, const Heads<const T>& k, const Heads<const T>& v, const Heads<const T>& d_o, const BwdArgs& w,
              const Heads<T>& dq, hipStream_t st) {
    const UnionSpace space(a, KeyTiles<T, DP, KW>::BYTES);
    static uint64_t allowed = 0;
    if (int e = allow_lds(reinterpret_cast<const void*>(&k_attention_dq<T, DP, KW>), LDS_BYTES, allowed)) return e;
    const int tiles = (int)cdiv(a.Tq, COLS / a.R);
    k_attention_dq<T, DP, KW><<<(unsigned)(tiles * a.B * a.G), ROW_THREADS, space.total, st>>>(a, plan, space, tiles, q, k, v, d_o, w.lse, w.delta, dq);
    MST_LAUNCH_CHECK();
    return MST_OK;
}

// f(DP, parts of 32 keys of a block)
template <typename F>
int with_sizes(const AttentionArgs& a, F&& f) {
    auto block = [&](auto dp) {
        if (a.BK == 32) return f(dp, std::integral_constant<int, 1>{});
        if (a.BK == 64) return f(dp, std::integral_constant<int, 2>{});
        return f(dp, std::integral_constant<int, 4>{});
    };
    return a.D <= 64 ? block(std::integral_constant<int, 64>{}) : block(std::integral_constant<int, 128>{});
}

}  // namespace
}  // namespace mst

extern "C" size_t mst_block_attention_workspace_bytes(const mst_attention_shape* s, int backward) {
    using namespace mst;
    if (check_attention(s)) return 0;
    return backward ? bwd_space(s).total : 256;
}

extern "C" int mst_block_attention_bwd(const mst_attention_shape* s, const mst_heads* q, const mst_heads* k, const mst_heads* v, const void* plan_dev,
                                       const mst_heads* o, const float* lse, const mst_heads* d_o, const mst_heads* dq, const mst_heads* dk, const mst_heads* dv,
                                       void* ws, size_t ws_bytes, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    if (s->batch == 0 || (s->queries == 0 && s->keys == 0)) return MST_OK;          // (empty buffers may be null)
    const struct { const mst_heads* v; bool key, written; } views[] = {{q, false, false}, {k, true, false}, {v, true, false}, {o, false, false}, {d_o, false, false}, {dq, false, true}, {dk, true, true}, {dv, true, true}};
    for (const auto& x : views)
        if (int e = x.key ? check_keys(s, x.v, x.written) : check_heads(x.v, s->batch, s->queries, s->heads, s->type, x.written)) return e;
    if ((s->queries > 0 && (!plan_dev || !lse)) || !ws || !aligned16(plan_dev) || !aligned16(lse) || !aligned16(ws)) return MST_ERR_ARG;
    const BwdSpace sp = bwd_space(s);
    if (ws_bytes < sp.total) return MST_ERR_WORKSPACE;
    const AttentionArgs a = attention_args(s);
    const Plan plan = carve_plan(plan_dev, a);
    const Lists lists = carve_lists(ws, a, sp.group);
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* base = static_cast<char*>(ws) + sp.lists;
    const BwdArgs w{lse, reinterpret_cast<float*>(base), reinterpret_cast<float*>(base + sp.delta), reinterpret_cast<float*>(base + sp.delta + sp.dkv)};
    int status = MST_OK;
    with_type(s->type, [&](auto type) {
        using T = decltype(type);
        const Heads<const T> qh = heads_of<const T>(q), kh = heads_of<const T>(k), vh = heads_of<const T>(v), oh = heads_of<const T>(o), doh = heads_of<const T>(d_o);
        const Heads<T> dqh = heads_of<T>(dq), dkh = heads_of<T>(dk), dvh = heads_of<T>(dv);
        if (a.Tq > 0) {
            float* delta = reinterpret_cast<float*>(base);
            const int64_t rows = (int64_t)a.Tq * a.H;
            if (a.D <= 64) k_attention_delta<T, 8><<<dim3((unsigned)cdiv(rows, 32), (unsigned)a.B), 256, 0, st>>>(a, oh, doh, delta);
            else k_attention_delta<T, 16><<<dim3((unsigned)cdiv(rows, 16), (unsigned)a.B), 256, 0, st>>>(a, oh, doh, delta);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) {
                g_last_hip_error = (int)e;
                status = MST_ERR_HIP;
                return;
            }
        }
        status = with_sizes(a, [&](auto dp, auto kp) {
            constexpr int DP = decltype(dp)::value, KP = decltype(kp)::value;
            if (a.S > 0)
                if (int e = launch_dkv<T, DP, KP>(a, plan, lists, sp, qh, kh, vh, doh, dkh, dvh, w, st)) return e;
            return a.Tq == 0 ? (int)MST_OK : launch_dq<T, DP, keys_at_once<T>(KP * 32)>(a, plan, qh, kh, vh, doh, w, dqh, st);
        });
    });
    return status;
}
