// Norm of the query and key heads and their rotation by position, forward and backward (mst_qk_norm_rotate).
//
// A head vector lies in one group of lanes, eight components to a lane: the mean of its squares is a sum over the
// group, and each value is read and written once.  Bound by memory at ten operations a value; few tokens by latency.
// The backward needs no more of the forward than x: with r = 1 / sqrt(mean x^2 + eps), dn the gradient rotated back and
// g = dn weight,  dx = r (g - x r^2 mean(g x)),  dweight = sum over the vectors of dn x r.  A lane meets the same
// components in all its vectors and keeps their sums in registers; a workgroup adds its lanes and writes one row, and a
// second launch adds the rows in order: the same sums in the same order every time.
#include "heads.h"

namespace mst {
namespace {

constexpr int NORM_THREADS = 256;
constexpr int NORM_BLOCKS = 1024;        // workgroups of the backward: rows of the weights' partial sums, at most

struct NormArgs {
    int64_t n;                           // vectors: batch x tokens x heads
    int tokens, heads, D, rotated, table_rows;
    float eps, inv_d;
    const float* weight;
    const float* table;
    const int* positions;
};

// the eight components of a lane after the rotation: x[e] of component i0 + e; other(i) = component i of the same vector
template <bool INTERLEAVED, bool BACK, typename F>
__device__ inline void rotate8(float (&x)[8], int i0, int rotated, const float* __restrict__ row, F&& other) {
    const int half = rotated >> 1;
    if (INTERLEAVED) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const int i = i0 + e;
            if (i >= rotated) break;
            const float c = row[i >> 1], s = BACK ? -row[half + (i >> 1)] : row[half + (i >> 1)];
            const float a = x[e], b = x[e + 1];
            x[e] = a * c - b * s;
            x[e + 1] = a * s + b * c;
        }
    } else {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = i0 + e;
            o[e] = i < rotated ? other(i < half ? i + half : i - half) : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = i0 + e;
            if (i >= rotated) break;
            const bool first = i < half;
            const float c = row[first ? i : i - half];
            float s = row[half + (first ? i : i - half)];
            if (BACK) s = -s;
            x[e] = first ? x[e] * c - o[e] * s : o[e] * s + x[e] * c;
        }
    }
}

template <int LANES, bool INTERLEAVED, typename TX, typename TY>
__device__ inline void norm_one(const NormArgs& a, const Heads<const TX>& x, const Heads<TY>& y, int64_t v, int lane) {
    const int64_t token = v / a.heads;
    const int h = (int)(v - token * a.heads), b = (int)(token / a.tokens), i0 = lane * 8;
    const int t = (int)(token - (int64_t)b * a.tokens);
    const bool mine = i0 < a.D;
    float xs[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const TX* px = x.at(b, t, h);
    if (mine) load8(px + i0, xs);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += xs[e] * xs[e];
    const float r = 1.f / sqrtf(lanes_sum<LANES>(sum) * a.inv_d + a.eps);
    if (!mine) return;
    float n[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) n[e] = xs[e] * r * (a.weight ? a.weight[i0 + e] : 1.f);
    if (i0 < a.rotated) {
        const int p = min(max(a.positions ? a.positions[token] : t, 0), a.table_rows - 1);
        rotate8<INTERLEAVED, false>(n, i0, a.rotated, a.table + (int64_t)p * a.rotated,
                                    [&](int i) { return to_float(px[i]) * r * (a.weight ? a.weight[i] : 1.f); });
    }
    store8(y.at(b, t, h) + i0, n);
}

// workgroups 0 .. q_blocks - 1 take the queries, the others the keys
template <int LANES, bool INTERLEAVED, typename TX, typename TY>
__global__ __launch_bounds__(NORM_THREADS) void k_norm_rotate(NormArgs qa, Heads<const TX> qx, Heads<TY> qy, int q_blocks,
                                                              NormArgs ka, Heads<const TX> kx, Heads<TY> ky) {
    constexpr int PER = NORM_THREADS / LANES;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const bool is_q = (int)blockIdx.x < q_blocks;
    const NormArgs& a = is_q ? qa : ka;
    const int64_t v = (int64_t)(is_q ? blockIdx.x : blockIdx.x - q_blocks) * PER + group;
    if (v >= a.n) return;
    if (is_q) norm_one<LANES, INTERLEAVED>(qa, qx, qy, v, lane);
    else norm_one<LANES, INTERLEAVED>(ka, kx, ky, v, lane);
}

template <int LANES, bool INTERLEAVED, typename TX, typename TY>
__device__ inline void norm_back(const NormArgs& a, const Heads<const TX>& x, const Heads<const TY>& dy, const Heads<TX>& dx, int64_t v, int lane, float (&dw)[8]) {
    const int64_t token = v / a.heads;
    const int h = (int)(v - token * a.heads), b = (int)(token / a.tokens), i0 = lane * 8;
    const int t = (int)(token - (int64_t)b * a.tokens);
    const bool mine = i0 < a.D;
    float xs[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, dn[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const TY* py = dy.at(b, t, h);
    if (mine) {
        load8(x.at(b, t, h) + i0, xs);
        load8(py + i0, dn);
        if (i0 < a.rotated) {
            const int p = min(max(a.positions ? a.positions[token] : t, 0), a.table_rows - 1);
            rotate8<INTERLEAVED, true>(dn, i0, a.rotated, a.table + (int64_t)p * a.rotated, [&](int i) { return to_float(py[i]); });
        }
    }
    float sum = 0.f, dot = 0.f, g[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        sum += xs[e] * xs[e];
        g[e] = mine && a.weight ? dn[e] * a.weight[i0 + e] : dn[e];
        dot += g[e] * xs[e];
    }
    const float r = 1.f / sqrtf(lanes_sum<LANES>(sum) * a.inv_d + a.eps);
    const float c = lanes_sum<LANES>(dot) * a.inv_d * r * r;
    if (!mine) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        dw[e] += dn[e] * xs[e] * r;
        g[e] = r * (g[e] - xs[e] * c);
    }
    store8(dx.at(b, t, h) + i0, g);
}

template <int LANES, bool INTERLEAVED, typename TX, typename TY>
__global__ __launch_bounds__(NORM_THREADS) void k_norm_rotate_bwd(NormArgs qa, Heads<const TX> qx, Heads<const TY> qdy, Heads<TX> qdx, int q_blocks,
                                                                  NormArgs ka, Heads<const TX> kx, Heads<const TY> kdy, Heads<TX> kdx,
                                                                  float* __restrict__ partial) {
    constexpr int PER = NORM_THREADS / LANES;
    __shared__ float sums[PER][LANES * 8 + 1];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const bool is_q = (int)blockIdx.x < q_blocks;
    const int block = is_q ? blockIdx.x : blockIdx.x - q_blocks, blocks = is_q ? q_blocks : gridDim.x - q_blocks;
    float dw[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int64_t n = is_q ? qa.n : ka.n, step = (int64_t)blocks * PER;
    for (int64_t v = (int64_t)block * PER + group; v < n; v += step) {   // (the lanes of a group leave together)
        if (is_q) norm_back<LANES, INTERLEAVED>(qa, qx, qdy, qdx, v, lane, dw);
        else norm_back<LANES, INTERLEAVED>(ka, kx, kdy, kdx, v, lane, dw);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[group][lane * 8 + e] = dw[e];
    __syncthreads();
    for (int i = threadIdx.x; i < qa.D; i += NORM_THREADS) {
        float s = 0.f;
        for (int j = 0; j < PER; ++j) s += sums[j][i];
        partial[(int64_t)blockIdx.x * qa.D + i] = s;
    }
}

// a workgroup adds one component over the rows: block (i, side)
__global__ __launch_bounds__(256) void k_norm_weight_sums(const float* __restrict__ partial, int D, int q_rows, int rows, float* __restrict__ dq,
                                                          float* __restrict__ dk) {
    __shared__ float part[4];
    float* out = blockIdx.y ? dk : dq;
    if (!out) return;
    const int r0 = blockIdx.y ? q_rows : 0, r1 = blockIdx.y ? rows : q_rows;
    float s = 0.f;
    for (int r = r0 + threadIdx.x; r < r1; r += 256) s += partial[(int64_t)r * D + blockIdx.x];
    s = lanes_sum<64>(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) out[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
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
    return {(int64_t)s->batch * s->tokens * heads, s->tokens, heads, s->head_dim, s->rotated, s->table_rows, s->eps, 1.f / (float)s->head_dim, weight, table, positions};
}

// f(lanes, interleaved, TX, TY) with the constants that the shape needs
template <typename F>
void norm_dispatch(const mst_qk_shape* s, F&& f) {
    auto types = [&](auto lanes, auto inter) {
        if (s->in_type == MST_F32) {
            if (s->out_type == MST_F32) f(lanes, inter, float{}, float{});
            else f(lanes, inter, float{}, bf16{});
        } else {
            if (s->out_type == MST_F32) f(lanes, inter, bf16{}, float{});
            else f(lanes, inter, bf16{}, bf16{});
        }
    };
    auto style = [&](auto lanes) {
        if (s->interleaved) types(lanes, std::true_type{});
        else types(lanes, std::false_type{});
    };
    switch (lanes_of(s->head_dim)) {
        case 4: style(std::integral_constant<int, 4>{}); break;
        case 8: style(std::integral_constant<int, 8>{}); break;
        case 16: style(std::integral_constant<int, 16>{}); break;
        default: style(std::integral_constant<int, 32>{}); break;
    }
}

struct NormGrid { int64_t q, k; };
NormGrid norm_blocks(const mst_qk_shape* s, bool backward) {
    const int64_t per = NORM_THREADS / lanes_of(s->head_dim), rows = (int64_t)s->batch * s->tokens;
    NormGrid g{cdiv(rows * s->heads, per), cdiv(rows * s->kv_heads, per)};
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
    norm_dispatch(s, [&](auto lanes, auto inter, auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        k_norm_rotate<decltype(lanes)::value, decltype(inter)::value, TX, TY><<<(unsigned)(g.q + g.k), NORM_THREADS, 0, st>>>(
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
        norm_dispatch(s, [&](auto lanes, auto inter, auto tx, auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            k_norm_rotate_bwd<decltype(lanes)::value, decltype(inter)::value, TX, TY><<<(unsigned)(g.q + g.k), NORM_THREADS, 0, st>>>(
                qa, heads_of<const TX>(q), heads_of<const TY>(dq_out), heads_of<TX>(dq_in), (int)g.q, ka, heads_of<const TX>(k), heads_of<const TY>(dk_out),
                heads_of<TX>(dk_in), partial);
        });
    MST_LAUNCH_CHECK();
    if (dqw || dkw) {                     // (with no vectors: zeros)
        k_norm_weight_sums<<<dim3((unsigned)s->head_dim, 2), 256, 0, st>>>(partial, s->head_dim, (int)g.q, (int)(g.q + g.k), dqw, dkw);
        MST_LAUNCH_CHECK();
    }
    return MST_OK;
}
