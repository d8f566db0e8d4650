// Norm of the query and key heads and their rotation by position, forward and backward (mst_qk_norm_rotate).
//
// A head vector lies in one group of lanes, two quads of components to a lane, such that a lane has both components of its
// pairs: the rotation needs no other lane, the mean of the squares is a sum over the group, and each value is read and
// written once.  A group takes two heads of one token in a row, so that the angles and weights are read once for them and
// their loads are on the way together.  Bound by memory at ten operations a value; few tokens by latency.
// Measured: 8 x 1024 tokens of 20 + 20 heads of 64, fp32 to bfloat16, 126 MB, 22 us back to back (some of it from the last level's cache; a copy
// of 1 GiB runs at 5.1 TB/s, 25 us for as much).
// The backward needs no more of the forward than x: with r = 1 / sqrt(mean x^2 + eps), dn the gradient rotated back and
// g = dn weight,  dx = r (g - x r^2 mean(g x)),  dweight = sum over the vectors of dn x r.  A lane meets the same
// components in all its vectors and keeps their sums in registers; a workgroup adds its lanes and writes one row, and a
// second launch adds the rows in order: the same sums in the same order every time.
#include "heads.h"

namespace mst {
namespace {

constexpr int NORM_THREADS = 256;
// Workgroups of the backward, at most: rows of the weights' partial sums.  (16 x 1024 tokens of 16 + 16 heads of 64: 41.7 us with 1024 of them, 44.0
// with 2048, 46.0 with 4096; 3 x 1531 of 16 + 4 heads of 128 in fp32 28.1, 30.0 and 34.9)
constexpr int NORM_BLOCKS = 1024;
// Heads of a token that a group takes: with one the angles are read for every head, with more the registers let fewer groups be on their way.  (forward
// of 8 x 1024 tokens of 20 + 20 heads, one, two, four, eight heads: 24.0, 21.8, 23.2, 23.4 us; the first backward above 46.2, 41.7, 49.1, 69.3; 32 single
// tokens of 12 + 12 heads 3.6, 3.8, 4.6, 6.3)
constexpr int NORM_HEADS = 2;

// which components a lane has.  HALVES: pairs (i, i + rotated / 2), whole quads of them; PAIRS: (2i, 2i + 1); APART: pairs
// (i, i + rotated / 2) where rotated / 2 is no multiple of 4, the other component read where it lies.
enum Style { HALVES, PAIRS, APART };

struct NormArgs {
    int64_t items;                       // groups' work: batch x tokens x parts of the heads
    int tokens, heads, parts, D, rotated, table_rows;
    float eps, inv_d;
    const float* weight;
    const float* table;
    const int* positions;
};

// the components of a lane and what stays the same over the heads of a token
template <Style S>
struct Lane {
    int a, b, angle;                     // first components of its two quads; index of its four angles
    bool mine, turns;
    __device__ Lane(const NormArgs& n, int lane) {
        const int pairs = S == HALVES ? n.rotated / 8 : 0;     // lanes with quads of both halves
        a = lane < pairs ? 4 * lane : n.rotated * (S == HALVES) + 8 * (lane - pairs);
        b = lane < pairs ? a + n.rotated / 2 : a + 4;
        mine = a < n.D;                  // (head_dim and, in HALVES, rotated are whole eights)
        angle = 4 * lane;
        turns = mine && (S == HALVES ? lane < pairs : a < n.rotated);
    }
};
struct Angles {
    float cos[4], sin[4];
};
template <bool BACK, Style S>
__device__ inline Angles angles_of(const NormArgs& n, const Lane<S>& l, int64_t token, int t) {
    Angles r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.cos[i] = 1.f, r.sin[i] = 0.f;
    if (S == APART || !l.turns) return r;
    const int half = n.rotated >> 1, p = min(max(n.positions ? n.positions[token] : t, 0), n.table_rows - 1);
    const float* row = n.table + (int64_t)p * n.rotated + l.angle;
    if ((half & 3) == 0) {               // rows, and the sines in them, at 16 bytes
        const float4 c = *reinterpret_cast<const float4*>(row), s = *reinterpret_cast<const float4*>(row + half);
        r.cos[0] = c.x; r.cos[1] = c.y; r.cos[2] = c.z; r.cos[3] = c.w;
        r.sin[0] = s.x; r.sin[1] = s.y; r.sin[2] = s.z; r.sin[3] = s.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (l.angle + i < half) r.cos[i] = row[i], r.sin[i] = row[half + i];
    }
    if (BACK)
#pragma unroll
        for (int i = 0; i < 4; ++i) r.sin[i] = -r.sin[i];
    return r;
}
template <Style S>
__device__ inline void turn(float (&x)[8], const Angles& w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float &u = x[S == HALVES ? i : 2 * i], &v = x[S == HALVES ? 4 + i : 2 * i + 1];
        const float n = u * w.cos[i] - v * w.sin[i];
        v = u * w.sin[i] + v * w.cos[i];
        u = n;
    }
}
// APART: component(i) of the vector before the rotation
template <bool BACK, typename F>
__device__ inline void turn_apart(float (&x)[8], const NormArgs& n, const Lane<APART>& l, int64_t token, int t, F&& component) {
    const int half = n.rotated >> 1, p = min(max(n.positions ? n.positions[token] : t, 0), n.table_rows - 1);
    const float* row = n.table + (int64_t)p * n.rotated;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = l.a + e;
        y[e] = x[e];
        if (i >= n.rotated) continue;
        const bool first = i < half;
        const float o = component(first ? i + half : i - half), c = row[first ? i : i - half];
        float s = row[first ? half + i : i];
        if (BACK) s = -s;
        y[e] = first ? x[e] * c - o * s : o * s + x[e] * c;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = y[e];
}

__device__ inline void load4(const float* p, float* x) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
}
__device__ inline void load4(const bf16* p, float* x) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    x[0] = __uint_as_float(a.x << 16); x[1] = __uint_as_float(a.x & 0xFFFF0000u);
    x[2] = __uint_as_float(a.y << 16); x[3] = __uint_as_float(a.y & 0xFFFF0000u);
}
template <typename T, Style S>
__device__ inline void load_lane(const T* p, const Lane<S>& l, float (&x)[8]) {
    if (S == HALVES) load4(p + l.a, x), load4(p + l.b, x + 4);
    else load8(p + l.a, x);
}
template <typename T, Style S>
__device__ inline void store_lane(T* p, const Lane<S>& l, const float (&x)[8]) {
    if (S == HALVES) store4(p + l.a, x[0], x[1], x[2], x[3]), store4(p + l.b, x[4], x[5], x[6], x[7]);
    else store8(p + l.a, x);
}

// where an item of work is
struct NormItem {
    int64_t token;
    int b, t, h0, h1;
    __device__ NormItem(const NormArgs& n, int64_t item) {
        token = item / n.parts;
        h0 = (int)(item - token * n.parts) * NORM_HEADS;
        h1 = min(h0 + NORM_HEADS, n.heads);
        b = (int)(token / n.tokens);
        t = (int)(token - (int64_t)b * n.tokens);
    }
};

template <int LANES, Style S, typename TX, typename TY>
__device__ inline void norm_item(const NormArgs& n, const Heads<const TX>& x, const Heads<TY>& y, int64_t item, int lane) {
    const Lane<S> l(n, lane);
    const NormItem it(n, item);
    float w[8], xs[NORM_HEADS][8];
#pragma unroll
    for (int i = 0; i < NORM_HEADS; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) xs[i][e] = 0.f;
        if (l.mine && it.h0 + i < it.h1) load_lane(x.at(it.b, it.t, it.h0 + i), l, xs[i]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.f;
    if (l.mine && n.weight) load_lane(n.weight, l, w);
    const Angles angles = angles_of<false>(n, l, it.token, it.t);
#pragma unroll
    for (int i = 0; i < NORM_HEADS; ++i) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += xs[i][e] * xs[i][e];
        const float r = 1.f / sqrtf(lanes_sum<LANES>(sum) * n.inv_d + n.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) xs[i][e] *= r * w[e];
        if constexpr (S != APART) turn<S>(xs[i], angles);
        else if (l.turns && it.h0 + i < it.h1) {
            const TX* px = x.at(it.b, it.t, it.h0 + i);
            turn_apart<false>(xs[i], n, l, it.token, it.t, [&](int c) { return to_float(px[c]) * (r * (n.weight ? n.weight[c] : 1.f)); });
        }
    }
#pragma unroll
    for (int i = 0; i < NORM_HEADS; ++i)
        if (l.mine && it.h0 + i < it.h1) store_lane(y.at(it.b, it.t, it.h0 + i), l, xs[i]);
}

// workgroups 0 .. q_blocks - 1 take the queries, the others the keys
template <int LANES, Style S, typename TX, typename TY>
__global__ __launch_bounds__(NORM_THREADS) void k_norm_rotate(NormArgs qa, Heads<const TX> qx, Heads<TY> qy, int q_blocks,
                                                              NormArgs ka, Heads<const TX> kx, Heads<TY> ky) {
    constexpr int PER = NORM_THREADS / LANES;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const bool is_q = (int)blockIdx.x < q_blocks;
    const int64_t item = (int64_t)(is_q ? blockIdx.x : blockIdx.x - q_blocks) * PER + group;
    if (item >= (is_q ? qa.items : ka.items)) return;          // (the lanes of a group leave together)
    if (is_q) norm_item<LANES, S>(qa, qx, qy, item, lane);
    else norm_item<LANES, S>(ka, kx, ky, item, lane);
}

template <int LANES, Style S, typename TX, typename TY>
__device__ inline void norm_back(const NormArgs& n, const Heads<const TX>& x, const Heads<const TY>& dy, const Heads<TX>& dx, int64_t first, int64_t step, int lane,
                                 float (&dw)[8]) {
    const Lane<S> l(n, lane);
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.f;
    if (l.mine && n.weight) load_lane(n.weight, l, w);
    for (int64_t item = first; item < n.items; item += step) {
        const NormItem it(n, item);
        float xs[NORM_HEADS][8], dn[NORM_HEADS][8];
#pragma unroll
        for (int i = 0; i < NORM_HEADS; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) xs[i][e] = dn[i][e] = 0.f;
            if (l.mine && it.h0 + i < it.h1) {
                load_lane(x.at(it.b, it.t, it.h0 + i), l, xs[i]);
                load_lane(dy.at(it.b, it.t, it.h0 + i), l, dn[i]);
            }
        }
        const Angles angles = angles_of<true>(n, l, it.token, it.t);
#pragma unroll
        for (int i = 0; i < NORM_HEADS; ++i) {
            if constexpr (S != APART) turn<S>(dn[i], angles);
            else if (l.turns && it.h0 + i < it.h1) {
                const TY* py = dy.at(it.b, it.t, it.h0 + i);
                turn_apart<true>(dn[i], n, l, it.token, it.t, [&](int c) { return to_float(py[c]); });
            }
            float sum = 0.f, dot = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum += xs[i][e] * xs[i][e];
                dot += dn[i][e] * w[e] * xs[i][e];
            }
            const float r = 1.f / sqrtf(lanes_sum<LANES>(sum) * n.inv_d + n.eps);
            const float c = lanes_sum<LANES>(dot) * n.inv_d * r * r;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[e] += it.h0 + i < it.h1 ? dn[i][e] * xs[i][e] * r : 0.f;        // (r of a vector that is not there may be infinite)
                dn[i][e] = r * (dn[i][e] * w[e] - xs[i][e] * c);
            }
        }
#pragma unroll
        for (int i = 0; i < NORM_HEADS; ++i)
            if (l.mine && it.h0 + i < it.h1) store_lane(dx.at(it.b, it.t, it.h0 + i), l, dn[i]);
    }
}

template <int LANES, Style S, typename TX, typename TY>
__global__ __launch_bounds__(NORM_THREADS) void k_norm_rotate_bwd(NormArgs qa, Heads<const TX> qx, Heads<const TY> qdy, Heads<TX> qdx, int q_blocks,
                                                                  NormArgs ka, Heads<const TX> kx, Heads<const TY> kdy, Heads<TX> kdx,
                                                                  float* __restrict__ partial) {
    constexpr int PER = NORM_THREADS / LANES;
    __shared__ float sums[PER][LANES * 8 + 1];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const bool is_q = (int)blockIdx.x < q_blocks;
    const int block = is_q ? blockIdx.x : blockIdx.x - q_blocks, blocks = is_q ? q_blocks : gridDim.x - q_blocks;
    float dw[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int64_t first = (int64_t)block * PER + group, step = (int64_t)blocks * PER;
    if (is_q) norm_back<LANES, S>(qa, qx, qdy, qdx, first, step, lane, dw);
    else norm_back<LANES, S>(ka, kx, kdy, kdx, first, step, lane, dw);
    const Lane<S> l(qa, lane);
    if (l.mine)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[group][l.a + e] = dw[e], sums[group][l.b + e] = dw[4 + e];
    __syncthreads();
    for (int i = threadIdx.x; i < qa.D; i += NORM_THREADS) {
        float s = 0.f;
        for (int j = 0; j < PER; ++j) s += sums[j][i];
        partial[(int64_t)blockIdx.x * qa.D + i] = s;
    }
}

// rows of the partial sums added: workgroup (eight components, side), 32 rows at a time
__global__ __launch_bounds__(256) void k_norm_weight_sums(const float* __restrict__ partial, int D, int q_rows, int rows, float* __restrict__ dq,
                                                          float* __restrict__ dk) {
    __shared__ float part[32][8];
    float* out = blockIdx.y ? dk : dq;
    if (!out) return;
    const int r0 = blockIdx.y ? q_rows : 0, r1 = blockIdx.y ? rows : q_rows, c = threadIdx.x & 7, g = threadIdx.x >> 3;
    float s = 0.f;
#pragma unroll 8
    for (int r = r0 + g; r < r1; r += 32) s += partial[(int64_t)r * D + blockIdx.x * 8 + c];
    part[g][c] = s;
    __syncthreads();
    if (g == 0) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += part[i][c];
        out[blockIdx.x * 8 + c] = s;
    }
}

int lanes_of(int D) { return D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32; }

int check_shape(const mst_qk_shape* s) {
    if (!s || !is_type(s->in_type) || !is_type(s->out_type) || !(s->eps >= 0.f) || !(s->eps <= 1e30f)) return MST_ERR_ARG;
    if (s->batch < 0 || s->tokens < 0 || s->heads < 0 || s->kv_heads < 0 || s->heads > HEADS_MAX || s->kv_heads > HEADS_MAX) return MST_ERR_SHAPE;
    if (s->head_dim < 8 || s->head_dim > 256 || s->head_dim % 8 != 0) return MST_ERR_SHAPE;
    if (s->rotated < 0 || s->rotated > s->head_dim || s->rotated % 2 != 0 || (s->rotated > 0 && s->table_rows < 1)) return MST_ERR_SHAPE;
    // a workgroup takes eight vectors or more: 2^31 of them at most
    if ((int64_t)s->batch * s->tokens > (int64_t(1) << 33) / std::max<int64_t>(1, (int64_t)s->heads + s->kv_heads)) return MST_ERR_SHAPE;
    return MST_OK;
}

NormArgs norm_args(const mst_qk_shape* s, int heads, const float* weight, const float* table, const int* positions) {
    const int parts = (int)cdiv(heads, NORM_HEADS);
    return {(int64_t)s->batch * s->tokens * parts, s->tokens, heads, parts, s->head_dim, s->rotated, s->table_rows, s->eps, 1.f / (float)s->head_dim, weight, table, positions};
}

// f(lanes, style, TX, TY) with the constants that the shape needs
template <typename F>
void norm_dispatch(const mst_qk_shape* s, F&& f) {
    auto types = [&](auto lanes, auto style) {
        if (s->in_type == MST_F32) {
            if (s->out_type == MST_F32) f(lanes, style, float{}, float{});
            else f(lanes, style, float{}, bf16{});
        } else {
            if (s->out_type == MST_F32) f(lanes, style, bf16{}, float{});
            else f(lanes, style, bf16{}, bf16{});
        }
    };
    auto with_style = [&](auto lanes) {
        if (s->interleaved) types(lanes, std::integral_constant<Style, PAIRS>{});
        else if (s->rotated % 8 == 0) types(lanes, std::integral_constant<Style, HALVES>{});
        else types(lanes, std::integral_constant<Style, APART>{});
    };
    switch (lanes_of(s->head_dim)) {
        case 4: with_style(std::integral_constant<int, 4>{}); break;
        case 8: with_style(std::integral_constant<int, 8>{}); break;
        case 16: with_style(std::integral_constant<int, 16>{}); break;
        default: with_style(std::integral_constant<int, 32>{}); break;
    }
}

struct NormGrid { int64_t q, k; };
NormGrid norm_blocks(const mst_qk_shape* s, bool backward) {
    const int64_t per = NORM_THREADS / lanes_of(s->head_dim), rows = (int64_t)s->batch * s->tokens;
    NormGrid g{cdiv(rows * cdiv(s->heads, NORM_HEADS), per), cdiv(rows * cdiv(s->kv_heads, NORM_HEADS), per)};
    if (backward && g.q + g.k > NORM_BLOCKS) {      // in proportion, one at least for each side that has vectors
        const int64_t q = g.k == 0 ? NORM_BLOCKS : std::min<int64_t>(NORM_BLOCKS - 1, std::max<int64_t>(g.q > 0, g.q * NORM_BLOCKS / (g.q + g.k)));
        g = {std::min(g.q, q), std::min(g.k, NORM_BLOCKS - q)};
    }
    return g;
}

int check_inputs(const mst_qk_shape* s, const mst_heads* q, const mst_heads* k, const float* qw, const float* kw, const float* table, const int* positions) {
    if (int e = check_shape(s)) return e;
    const int64_t B = s->batch, T = s->tokens;
    if (s->heads > 0)
        if (int e = check_heads(q, B, T, s->heads, s->in_type, false)) return e;
    if (s->kv_heads > 0)
        if (int e = check_heads(k, B, T, s->kv_heads, s->in_type, false)) return e;
    if (s->rotated > 0 && !table) return MST_ERR_ARG;
    if (!aligned16(qw) || !aligned16(kw) || !aligned16(table) || !aligned16(positions)) return MST_ERR_ARG;
    return MST_OK;
}

const mst_heads NO_HEADS = {nullptr, 0, 0, 0};

}  // namespace
}  // namespace mst

extern "C" int mst_qk_norm_rotate(const mst_qk_shape* s, const mst_heads* q, const mst_heads* k, const float* qw, const float* kw, const float* table,
                                  const int32_t* positions, const mst_heads* q_out, const mst_heads* k_out, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_inputs(s, q, k, qw, kw, table, positions)) return e;
    if (s->heads > 0)
        if (int e = check_heads(q_out, s->batch, s->tokens, s->heads, s->out_type, true)) return e;
    if (s->kv_heads > 0)
        if (int e = check_heads(k_out, s->batch, s->tokens, s->kv_heads, s->out_type, true)) return e;
    if (!s->heads) q = q_out = &NO_HEADS;
    if (!s->kv_heads) k = k_out = &NO_HEADS;
    const NormGrid g = norm_blocks(s, false);
    if (g.q + g.k == 0) return MST_OK;
    const NormArgs qa = norm_args(s, s->heads, qw, table, positions), ka = norm_args(s, s->kv_heads, kw, table, positions);
    hipStream_t st = static_cast<hipStream_t>(stream);
    norm_dispatch(s, [&](auto lanes, auto style, auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        k_norm_rotate<decltype(lanes)::value, decltype(style)::value, TX, TY><<<(unsigned)(g.q + g.k), NORM_THREADS, 0, st>>>(
            qa, heads_of<const TX>(q), heads_of<TY>(q_out), (int)g.q, ka, heads_of<const TX>(k), heads_of<TY>(k_out));
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}

extern "C" size_t mst_qk_norm_rotate_workspace_bytes(const mst_qk_shape* s) {
    using namespace mst;
    if (check_shape(s)) return 0;
    const NormGrid g = norm_blocks(s, true);
    return align_up(std::max<size_t>(1, (size_t)(g.q + g.k)) * s->head_dim * sizeof(float));
}

extern "C" int mst_qk_norm_rotate_bwd(const mst_qk_shape* s, const mst_heads* q, const mst_heads* k, const float* qw, const float* kw, const float* table,
                                      const int32_t* positions, const mst_heads* dq_out, const mst_heads* dk_out, const mst_heads* dq_in,
                                      const mst_heads* dk_in, float* dqw, float* dkw, void* ws, size_t ws_bytes, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_inputs(s, q, k, qw, kw, table, positions)) return e;
    if (s->heads > 0) {
        if (int e = check_heads(dq_out, s->batch, s->tokens, s->heads, s->out_type, false)) return e;
        if (int e = check_heads(dq_in, s->batch, s->tokens, s->heads, s->in_type, true)) return e;
    }
    if (s->kv_heads > 0) {
        if (int e = check_heads(dk_out, s->batch, s->tokens, s->kv_heads, s->out_type, false)) return e;
        if (int e = check_heads(dk_in, s->batch, s->tokens, s->kv_heads, s->in_type, true)) return e;
    }
    if (!ws || !aligned16(ws) || !aligned16(dqw) || !aligned16(dkw)) return MST_ERR_ARG;
    if (ws_bytes < mst_qk_norm_rotate_workspace_bytes(s)) return MST_ERR_WORKSPACE;
    if (!s->heads) q = dq_out = dq_in = &NO_HEADS;
    if (!s->kv_heads) k = dk_out = dk_in = &NO_HEADS;
    const NormGrid g = norm_blocks(s, true);
    const NormArgs qa = norm_args(s, s->heads, qw, table, positions), ka = norm_args(s, s->kv_heads, kw, table, positions);
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* partial = static_cast<float*>(ws);
    if (g.q + g.k > 0)
        norm_dispatch(s, [&](auto lanes, auto style, auto tx, auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            k_norm_rotate_bwd<decltype(lanes)::value, decltype(style)::value, TX, TY><<<(unsigned)(g.q + g.k), NORM_THREADS, 0, st>>>(
                qa, heads_of<const TX>(q), heads_of<const TY>(dq_out), heads_of<TX>(dq_in), (int)g.q, ka, heads_of<const TX>(k), heads_of<const TY>(dk_out),
                heads_of<TX>(dk_in), partial);
        });
    MST_LAUNCH_CHECK();
    if (dqw || dkw) {                     // (with no vectors: zeros)
        k_norm_weight_sums<<<dim3((unsigned)(s->head_dim / 8), 2), 256, 0, st>>>(partial, s->head_dim, (int)g.q, (int)(g.q + g.k), dqw, dkw);
        MST_LAUNCH_CHECK();
    }
    return MST_OK;
}
