// Attention over selected blocks of keys, forward (mst_block_attention_fwd) and for single tokens (mst_block_attention_decode).
//
// Forward: rows that own their results walk the union of their blocks (block_rows.h).  With S^T = K Q^T a lane has the scores of one
// row, half of 32 keys, and its probabilities are at once the operand of O^T = V^T P^T; keys are read from LDS along their
// rows and values across them.  P is rounded to bfloat16 for that product where the heads are (its sum is not): the weights' error is
// that of the output's own rounding.
//
// A row that does not see a block of the union has the weight 2^-inf there.  That is 0 but where its product with a block that it has nothing to do with
// left fp32: those weights show as a sum that is no number, and are cleared.
//
// Measured: 32768 queries of 32 heads of 128 with 8 key heads, 16 blocks of 128 a query, 2.45 ms: 425 TFLOP/s of what the rows
// selected; 32 rows visit 28.4 blocks where a row has 15.5, so the matrix instructions do 780, of 1255 that a product of 8192 x 8192 x 8192 does
// on this card.  (Among passes that follow each other; the first ten after a pause take 2.4 to 3.1, 2.68 on average, as the clock moves.)  Matrix
// instructions are busy in 34 % of the clocks, the vector instructions (exponentials, maxima, roundings) in about as many, and a SIMD's two
// wavefronts overlap the two in part.  8192 queries of 20 heads of 64, 8 blocks of 64: 146 us; there 32 rows visit 27.4 blocks for 7.8.
#include "block_rows.h"

namespace mst {
namespace {

// The weights of a row are 2^(score - reference), the reference a maximum that is left behind until a score passes it by more than
// this: sums of weights stay far inside fp32, and the results are seldom scaled anew.  (8192 queries of 20 heads 133 us, 135 with 0; 2 x 4099 of 24
// heads of 128 with 8 key heads 128 and 133)
constexpr float SLACK = 8.f;

template <typename T, int DP, int KW>
__global__ __launch_bounds__(ROW_THREADS, (sizeof(T) * DP == 512 ? 1 : 2)) void k_attention_fwd(AttentionArgs a, Plan plan, UnionSpace space, int tiles, Heads<const T> q, Heads<const T> k,
                                                                  Heads<const T> v, Heads<T> o, float* __restrict__ lse) {
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
    // a positive factor, so that the highest product is the highest score: its sign goes to the query
    const float scale2 = fmaxf(fabsf(a.scale) * LOG2E, 1.17549435e-38f);
    Cursor cursor(a, rows, tok, there);
    const bool sees = there && cursor.next < a.nb;             // (the vector of a row that sees nothing may hold anything)
    Operand<T> qf[QC];
    const T* qp = q.at(b, there ? t : 0, there ? h : 0);
#pragma unroll
    for (int c = 0; c < QC; ++c) {
        qf[c] = sees && c * 16 + half * 8 < a.D ? load_operand(qp + c * 16 + half * 8) : zero_operand<T>();
        if (a.scale < 0.f) qf[c] = negated(qf[c]);
    }
    floatx16 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = zero16();
    float m = LOWEST, l = 0.f;
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
            const int limit = cursor.next == (int)(now & 0xFFFF) ? p - key0 : -1;          // the row sees the keys 0 .. limit of this part
            floatx16 s[ST];
#pragma unroll
            for (int st = 0; st < ST; ++st) {
                s[st] = zero16();
#pragma unroll
                for (int c = 0; c < QC; ++c)
                    if (worth<T>(c * 16, a.D)) s[st] = product32(along_row<T, DP>(tile, st * 32 + i32, c * 16 + half * 8), qf[c], s[st]);
            }
            if (__any(limit < KW - 1 && limit >= 0)) {         // some row sees some of these keys, not all
#pragma unroll
                for (int st = 0; st < ST; ++st)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (st * 32 + 8 * (r / 4) + 4 * half + r % 4 > limit) s[st][r] = -INFINITY;
            }
            float top = s[0][0];
#pragma unroll
            for (int e = 1; e < ST * 16; ++e) top = fmaxf(top, s[e / 16][e % 16]);
            top = apart<32>(top, [](float u, float w) { return fmaxf(u, w); }) * scale2;
            if (limit < 0) top = -INFINITY;
            if (__any(top > m + SLACK)) {
                const float to = fmaxf(m, top), f = exp2_fast(m - to);
                m = to;
                l *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[d][r] *= f;
            }
            const float less = limit < 0 ? INFINITY : m;       // a row that sees nothing here: weights 2^-inf
            const float before = l;
            Operand<T> pf[2 * ST];
#pragma unroll
            for (int u = 0; u < 2 * ST; ++u) {
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[e] = exp2_fast(__builtin_fmaf(s[u / 2][(u % 2) * 8 + e], scale2, -less));
                    l += w[e];
                }
                set_operand(pf[u], w);
            }
            // ... which are 0 but where a product that the row has nothing to do with left fp32: then its sum is no number
            if (__any(limit < 0 && l != l))
                if (limit < 0) {
                    l = before;
#pragma unroll
                    for (int u = 0; u < 2 * ST; ++u) pf[u] = zero_operand<T>();
                }
#pragma unroll
            for (int d = 0; d < DT; ++d)
                if (worth<T>(d * 32, a.D))
#pragma unroll
                    for (int u = 0; u < 2 * ST; ++u) acc[d] = product32(across_rows<T, DP>(tile + Tiles::TILE, u * 16, d * 32, lane), pf[u], acc[d]);
        }
        if (block_ends) cursor.pass(a, (int)(now & 0xFFFF));
    }
    if (!there) return;
    l = apart<32>(l, [](float u, float w) { return u + w; });
    const float scale = l == 0.f ? 0.f : 1.f / l;              // (a row without keys; not one whose sum is no number)
    T* po = o.at(b, t, h);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int c = d * 32 + 2 * r + 4 * half;
            if (c < a.D) store4(po + c, acc[d][r] * scale, acc[d][r + 1] * scale, acc[d][r + 2] * scale, acc[d][r + 3] * scale);
        }
    if (half == 0) lse[((int64_t)b * a.H + h) * a.Tq + t] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}

// ---- single tokens: a workgroup per (query, key head, RT of its heads); its wavefronts take pieces of the selected blocks in turn, the
// next piece on its way while they work on one.  A key is LANES lanes of eight components, so a wavefront reads 64 / LANES keys in
// a row; with one to four rows the products are no work for matrix instructions (the reads take longer) and every value stays
// in registers, in fp32, until the wavefronts are joined.  Bound by memory: 64 sequences, 8 key heads of 4 heads of 128, 16 blocks of 64 of
// up to 16384 tokens, 268 MB of keys and values, take 53 us (5.1 TB/s; part of them from the last level's cache).
template <typename T, int LANES, int RT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_attention_decode(AttentionArgs a, Heads<const T> q, Heads<const T> k, Heads<const T> v, const int* __restrict__ blocks,
                                                                  Heads<T> o, float* __restrict__ lse) {
    constexpr int KEYS = 64 / LANES, PIECE = sizeof(T) == 2 ? 32 : 16, STEPS = PIECE / KEYS;
    __shared__ float part[WAVES][RT][LANES * 8];
    __shared__ float part_m[WAVES][RT], part_l[WAVES][RT];
    __shared__ int list[SELECT_MAX];
    const int groups = (a.R + RT - 1) / RT, t = blockIdx.x / groups, r0 = (blockIdx.x - t * groups) * RT;
    const int bg = blockIdx.y, b = bg / a.G, g = bg % a.G, len = a.length(b), p = len - a.Tq + t;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % LANES, key_of = lane / LANES;
    const int own = p >= 0 ? p / a.BK : -1, at = min(c * 8, a.D - 8);          // (past head_dim: the last components again, met by zeros)
    const float scale2 = a.scale * LOG2E;
    // entries that count, one lane each: above all before them and up to the own block
    const int j = lane < a.NS ? blocks[((int64_t)bg * a.Tq + t) * a.NS + lane] : -1;
    int high = j >= 0 && j <= own ? j : -1;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(high, d);
        if (lane >= d) high = max(high, x);
    }
    const int before = __shfl_up(high, 1);
    const bool counts = j >= 0 && j <= own && (lane == 0 || j > before);
    const uint64_t valid = __ballot(counts);
    if (wave == 0 && counts) list[__popcll(valid & ((1ull << lane) - 1))] = j;
    float qs[RT][8], acc[RT][8], m[RT], l[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = LOWEST, l[r] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) qs[r][e] = acc[r][e] = 0.f;
        if (c * 8 < a.D && r0 + r < a.R) load8(q.at(b, t, g * a.R + r0 + r) + c * 8, qs[r]);
#pragma unroll
        for (int e = 0; e < 8; ++e) qs[r][e] *= scale2;
    }
    __syncthreads();
    const int per = a.BK / PIECE, pieces = __popcll(valid) * per;
    struct Piece { Operand<T> k[STEPS], v[STEPS]; };
    auto key_of_piece = [&](int n) { return list[n / per] * a.BK + n % per * PIECE; };
    auto fetch = [&](int n, Piece& x) {
        const int key0 = key_of_piece(n) + key_of;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) x.k[s] = load_operand(k.at(b, min(key0 + s * KEYS, p), g) + at);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) x.v[s] = load_operand(v.at(b, min(key0 + s * KEYS, p), g) + at);
    };
    auto work = [&](int n, const Piece& piece) {
        const int key0 = key_of_piece(n);
        if (key0 > p) return;                                  // (behind the query in its own block)
        float x[RT][STEPS], y[8];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            numbers(piece.k[s], y);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float d = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) d += qs[r][e] * y[e];
                d = lanes_sum<LANES>(d);
                x[r][s] = key0 + s * KEYS + key_of <= p ? d : -INFINITY;
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = x[r][0];
#pragma unroll
            for (int s = 1; s < STEPS; ++s) top = fmaxf(top, x[r][s]);
            auto higher = [](float u, float w) { return fmaxf(u, w); };
            if (LANES <= 8) top = higher(top, __shfl_xor(top, 8));
            top = apart<32>(apart<16>(top, higher), higher);
            const float to = fmaxf(m[r], top), f = exp2_fast(m[r] - to);
            m[r] = to;
            l[r] *= f;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[r][e] *= f;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                x[r][s] = exp2_fast(x[r][s] - to);
                l[r] += x[r][s];
            }
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            numbers(piece.v[s], y);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[r][e] += x[r][s] * y[e];
        }
    };
    Piece one, two;
    int n = wave;
    if (n < pieces) fetch(n, one);
    for (; n < pieces; n += 2 * WAVES) {
        if (n + WAVES < pieces) fetch(n + WAVES, two);
        work(n, one);
        if (n + 2 * WAVES < pieces) fetch(n + 2 * WAVES, one);
        if (n + WAVES < pieces) work(n + WAVES, two);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        auto add = [](float u, float w) { return u + w; };
        auto over_keys = [&](float u) {
            if (LANES <= 8) u += __shfl_xor(u, 8);
            return apart<32>(apart<16>(u, add), add);
        };
        l[r] = over_keys(l[r]);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[r][e] = over_keys(acc[r][e]);
        if (key_of == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) part[wave][r][c * 8 + e] = acc[r][e];
            if (c == 0) part_m[wave][r] = m[r], part_l[wave][r] = l[r];
        }
    }
    __syncthreads();
    for (int u = threadIdx.x; u < RT * LANES * 2; u += WAVES * 64) {          // four components of a head to a thread
        const int r = u / (LANES * 2), d = (u - r * (LANES * 2)) * 4;
        if (r0 + r >= a.R || d >= a.D) continue;
        float top = LOWEST, sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, part_m[w][r]);
        for (int w = 0; w < WAVES; ++w) {
            const float f = exp2f(part_m[w][r] - top);
            sum += part_l[w][r] * f;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] += part[w][r][d + e] * f;
        }
        const float n1 = sum == 0.f ? 0.f : 1.f / sum;
        store4(o.at(b, t, g * a.R + r0 + r) + d, x[0] * n1, x[1] * n1, x[2] * n1, x[3] * n1);
        if (d == 0 && lse) lse[((int64_t)b * a.H + g * a.R + r0 + r) * a.Tq + t] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
    }
}

}  // namespace
}  // namespace mst

extern "C" int mst_block_attention_fwd(const mst_attention_shape* s, const mst_heads* q, const mst_heads* k, const mst_heads* v, const void* plan_dev,
                                       const mst_heads* o, float* lse, void* ws, size_t ws_bytes, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    if (s->batch == 0 || s->queries == 0) return MST_OK;       // (empty buffers may be null)
    if (int e = check_heads(q, s->batch, s->queries, s->heads, s->type, false)) return e;
    if (int e = check_keys(s, k, false)) return e;
    if (int e = check_keys(s, v, false)) return e;
    if (int e = check_heads(o, s->batch, s->queries, s->heads, s->type, true)) return e;
    if (!plan_dev || !lse || !aligned16(plan_dev) || !aligned16(lse) || !aligned16(ws) || (!ws && ws_bytes > 0)) return MST_ERR_ARG;
    if (ws && ws_bytes < mst_block_attention_workspace_bytes(s, 0)) return MST_ERR_WORKSPACE;          // (nothing is kept there: none will do)
    const AttentionArgs a = attention_args(s);
    const Plan plan = carve_plan(plan_dev, a);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int tiles = (int)cdiv(a.Tq, COLS / a.R);
    int status = MST_OK;
    with_type(s->type, [&](auto type) {
        using T = decltype(type);
        auto launch = [&](auto dp, auto kw) {
            constexpr int DP = decltype(dp)::value, KW = decltype(kw)::value;
            const UnionSpace space(a, KeyTiles<T, DP, KW>::BYTES);
            static uint64_t allowed = 0;
            const void* kernel = reinterpret_cast<const void*>(&k_attention_fwd<T, DP, KW>);
            status = allow_lds(kernel, LDS_BYTES, allowed);
            if (status) return;
            k_attention_fwd<T, DP, KW><<<(unsigned)(tiles * a.B * a.G), ROW_THREADS, space.total, st>>>(a, plan, space, tiles, heads_of<const T>(q), heads_of<const T>(k), heads_of<const T>(v), heads_of<T>(o), lse);
        };
        auto width = [&](auto kw) {
            if (a.D <= 64) launch(std::integral_constant<int, 64>{}, kw);
            else launch(std::integral_constant<int, 128>{}, kw);
        };
        if (a.BK == 32) width(std::integral_constant<int, 32>{});
        else width(std::integral_constant<int, keys_at_once<T>(64)>{});
    });
    if (status) return status;
    MST_LAUNCH_CHECK();
    return MST_OK;
}

extern "C" int mst_block_attention_decode(const mst_attention_shape* s, const mst_heads* q, const mst_heads* k, const mst_heads* v, const int32_t* blocks,
                                          const mst_heads* o, float* lse, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    if (s->batch == 0 || s->queries == 0) return MST_OK;       // (empty buffers may be null)
    if (int e = check_heads(q, s->batch, s->queries, s->heads, s->type, false)) return e;
    if (int e = check_keys(s, k, false)) return e;
    if (int e = check_keys(s, v, false)) return e;
    if (int e = check_heads(o, s->batch, s->queries, s->heads, s->type, true)) return e;
    if (!blocks || !aligned16(blocks) || !aligned16(lse)) return MST_ERR_ARG;
    const AttentionArgs a = attention_args(s);
    hipStream_t st = static_cast<hipStream_t>(stream);
    with_type(s->type, [&](auto type) {
        using T = decltype(type);
        const Heads<const T> qh = heads_of<const T>(q), kh = heads_of<const T>(k), vh = heads_of<const T>(v);
        const Heads<T> oh = heads_of<T>(o);
        auto launch = [&](auto lanes, auto rt, auto waves) {
            constexpr int L = decltype(lanes)::value, RT = decltype(rt)::value, WAVES = decltype(waves)::value;
            k_attention_decode<T, L, RT, WAVES><<<dim3((unsigned)(cdiv(a.R, RT) * a.Tq), (unsigned)(a.B * a.G)), WAVES * 64, 0, st>>>(a, qh, kh, vh, blocks, oh, lse);
        };
        auto width = [&](auto rt, auto waves) {
            if (a.D <= 64) launch(std::integral_constant<int, 8>{}, rt, waves);
            else launch(std::integral_constant<int, 16>{}, rt, waves);
        };
        // Up to four heads to a workgroup, which then reads the keys once for them (of 8 to 64 heads of a key head, 2 to 16 workgroups read
        // them; of three, a quarter of the work is for nobody), but one for each CU if there are heads (one sequence, 8 key heads of 4, 16 blocks
        // of 64: 21.5 us with four heads to a workgroup, 11.7 with one; below 256 (query, head) every head reads the keys for itself).  Eight wavefronts where workgroups are still too few for the card,
        // four where CUs hold several (that sequence 11.7 with eight, 12.6 with four; two key heads of 16, 32 blocks of 128: 31 and 39;
        // 64 sequences of 8 key heads of 4: 63 and 53).
        constexpr int CUS = 256;
        auto groups = [&](int rt) { return (int64_t)a.B * a.G * a.Tq * cdiv(a.R, rt); };
        int rt = a.R == 1 ? 1 : a.R == 2 ? 2 : 4;
        while (rt > 1 && groups(rt) < CUS) rt /= 2;
        if (groups(rt) < CUS) width(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{});
        else if (rt == 1) width(std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
        else if (rt == 2) width(std::integral_constant<int, 2>{}, std::integral_constant<int, 4>{});
        else width(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}
