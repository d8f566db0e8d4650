// Attention over selected blocks of keys, forward (mst_block_attention_fwd) and for single tokens (mst_block_attention_decode).
//
// Forward, from the lists of the plan: a wavefront keeps the keys of a block and its values, turned, in registers as operands
// of the matrix instructions and walks the rows (query, head) that selected the block, sixteen at a time.  With S^T = K Q^T
// a lane has the scores of one row and its probabilities are at once the operand of O^T = V^T P^T: the loop needs no LDS and no
// barrier, and its loads are the sixteen queries.  Each (row, block) leaves its sum of values, maximum and sum of
// weights in fp32; a second launch joins a row's blocks.  Work is in proportion to the pairs, whatever the rows select.
#include "block_attention.h"

namespace mst {
namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int FWD_THREADS = 256;

// keys that a wavefront of the forward holds: a block, or a part of one whose keys and values fit the registers
template <typename T, int DP> constexpr int keys_held() { return sizeof(T) == 4 && DP > 64 ? 32 : 64; }

// rows of the groups of (batch, key head) that one launch takes: their partial results stay near the caches
constexpr size_t PARTIAL_BYTES = size_t(256) << 20;

struct Partials {
    float* o;                            // [row-block][D]
    float2* ml;                          // [row-block] maximum (base 2) and sum
};

template <typename T, int DP, int KW>
__global__ __launch_bounds__(FWD_THREADS) void k_attention_fwd(AttentionArgs a, Plan plan, Heads<const T> q, Heads<const T> k, Heads<const T> v, int bg0, Partials out) {
    constexpr int KT = KW / 16, DC = DP / 32, DT = DP / 16, KS = KW / 32, ROW = TileRow<T, DP>::stride;
    __shared__ __align__(16) T vt[KW * ROW];
    const int bg = bg0 + blockIdx.y, b = bg / a.G, g = bg % a.G, parts = a.BK / KW;
    const int item = blockIdx.x / parts, part = blockIdx.x - item * parts;
    if (item >= plan.item_start[(int64_t)bg * (a.nb + 1) + a.nb]) return;
    const int2 it = plan.items[(int64_t)bg * plan.max_items + item];
    const int last = min(it.y + plan.item_pairs, plan.start[(int64_t)bg * (a.nb + 1) + it.x + 1]);
    const int len = a.length(b), key0 = it.x * a.BK + part * KW;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, quad = lane >> 4;

    Operand<T> kf[KT][DC];               // rows = keys
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            const int key = key0 + kt * 16 + i16, d = c * 32 + quad * 8;
            kf[kt][c] = key < len && d < a.D ? load_operand(k.at(b, key, g) + d) : zero_operand<T>();
        }
    for (int u = threadIdx.x; u < KW * (DP / 8); u += FWD_THREADS) {
        const int r = u / (DP / 8), d = (u % (DP / 8)) * 8;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (key0 + r < len && d < a.D) load8(v.at(b, key0 + r, g) + d, x);
        store8(&vt[r * ROW + d], x);
    }
    __syncthreads();
    Operand<T> vf[DT][KS];               // rows = components, contraction over the keys in the order of a product's rows
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int s = 0; s < KS; ++s) vf[dt][s] = across<ROW>(&vt[s * 32 * ROW + dt * 16], lane);

    const int rows = (last - it.y) * a.R;
    const int* list = plan.list + (int64_t)bg * a.Tq * a.NS;
    const int64_t pair0 = (int64_t)blockIdx.y * a.Tq * a.NS;
    const float scale2 = a.scale * LOG2E;
    for (int r0 = wave * 16; r0 < rows; r0 += FWD_THREADS / 4) {
        const int row = r0 + i16;
        const bool there = row < rows;
        const int e = there ? row / a.R : 0, h = there ? row - e * a.R : 0;
        const int pair = list[it.y + e], t = pair / a.NS;
        const T* qp = q.at(b, t, g * a.R + h);
        Operand<T> qf[DC];
#pragma unroll
        for (int c = 0; c < DC; ++c) qf[c] = c * 32 + quad * 8 < a.D ? load_operand(qp + c * 32 + quad * 8) : zero_operand<T>();
        floatx4 s[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            s[kt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < DC; ++c) s[kt] = product(kf[kt][c], qf[c], s[kt]);
        }
        const int limit = len - a.Tq + t - key0;               // the row sees the keys 0 .. limit of this part
        float m = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[kt][r] = kt * 16 + 4 * quad + r <= limit ? s[kt][r] * scale2 : -INFINITY;
                m = fmaxf(m, s[kt][r]);
            }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float base = m == -INFINITY ? 0.f : m;           // (a part without visible keys)
        float l = 0.f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[kt][r] = exp2f(s[kt][r] - base);
                l += s[kt][r];
            }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        Operand<T> pf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const float x[8] = {s[2 * ks][0], s[2 * ks][1], s[2 * ks][2], s[2 * ks][3], s[2 * ks + 1][0], s[2 * ks + 1][1], s[2 * ks + 1][2], s[2 * ks + 1][3]};
            set_operand(pf[ks], x);
        }
        const int64_t at = ((pair0 + pair) * a.R + h) * parts + part;
        float* po = out.o + at * a.D;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) o = product(vf[dt][ks], pf[ks], o);
            const int d = dt * 16 + 4 * quad;
            if (there && d < a.D) store4(po + d, o[0], o[1], o[2], o[3]);
        }
        if (there && quad == 0) out.ml[at] = make_float2(m, l);
    }
}

// joins the blocks of a row: LANES lanes of four components
template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_attention_join(AttentionArgs a, Plan plan, int parts, int bg0, Partials in, Heads<T> o, float* __restrict__ lse) {
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;    // (query, head) of a key head
    if (row >= (int64_t)a.Tq * a.R) return;
    const int t = (int)(row / a.R), h = (int)(row - (int64_t)t * a.R), bg = bg0 + blockIdx.y, b = bg / a.G, g = bg % a.G;
    const uint64_t valid = plan.valid[(int64_t)bg * a.Tq + t];
    const int64_t pair0 = (int64_t)blockIdx.y * a.Tq * a.NS + (int64_t)t * a.NS;
    float m = -INFINITY;
    for (uint64_t w = valid; w; w &= w - 1) {
        const int64_t at = ((pair0 + __ffsll((unsigned long long)w) - 1) * a.R + h) * parts;
        for (int p = 0; p < parts; ++p) m = fmaxf(m, in.ml[at + p].x);
    }
    float l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
    for (uint64_t w = valid; w; w &= w - 1) {
        const int64_t at = ((pair0 + __ffsll((unsigned long long)w) - 1) * a.R + h) * parts;
        for (int p = 0; p < parts; ++p) {
            const float2 ml = in.ml[at + p];
            if (ml.x == -INFINITY) continue;
            const float f = exp2f(ml.x - m);
            l += ml.y * f;
            if (lane * 4 < a.D) {
                const float4 y = *reinterpret_cast<const float4*>(in.o + (at + p) * a.D + lane * 4);
                x[0] += y.x * f; x[1] += y.y * f; x[2] += y.z * f; x[3] += y.w * f;
            }
        }
    }
    const float n = l == 0.f ? 0.f : 1.f / l;                  // (a row without keys; not one whose sum is no number)
    if (lane * 4 < a.D) store4(o.at(b, t, g * a.R + h) + lane * 4, x[0] * n, x[1] * n, x[2] * n, x[3] * n);
    if (lane == 0) lse[((int64_t)b * a.H + g * a.R + h) * a.Tq + t] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}

// ---- single tokens: a workgroup per (query, key head, RT of its heads), a wavefront per selected block at a time.  A key is LANES
// lanes of eight components, so a wavefront reads 64 / LANES keys in a row; with one to eight rows the products are no work
// for matrix instructions (the reads take longer) and every value stays in registers until the wavefronts are joined.
constexpr int DEC_THREADS = 512;
template <typename T, int LANES, int RT>
__global__ __launch_bounds__(DEC_THREADS) void k_attention_decode(AttentionArgs a, Heads<const T> q, Heads<const T> k, Heads<const T> v, const int* __restrict__ blocks,
                                                                  Heads<T> o, float* __restrict__ lse) {
    constexpr int KEYS = 64 / LANES, WAVES = DEC_THREADS / 64, STEPS = 32 / KEYS;    // 32 keys at a time
    __shared__ float part[WAVES][RT][LANES * 8];
    __shared__ float part_m[WAVES][RT], part_l[WAVES][RT];
    const int groups = (a.R + RT - 1) / RT, t = blockIdx.x / groups, r0 = (blockIdx.x - t * groups) * RT;
    const int bg = blockIdx.y, b = bg / a.G, g = bg % a.G, len = a.length(b), p = len - a.Tq + t;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane % LANES, key_of = lane / LANES;
    const bool mine = c * 8 < a.D;
    const int own = p >= 0 ? p / a.BK : -1;
    const int* row = blocks + ((int64_t)bg * a.Tq + t) * a.NS;
    float qs[RT][8], acc[RT][8], m[RT], l[RT];
    const float scale2 = a.scale * LOG2E;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) qs[r][e] = acc[r][e] = 0.f;
        if (mine && r0 + r < a.R) load8(q.at(b, t, g * a.R + r0 + r) + c * 8, qs[r]);
#pragma unroll
        for (int e = 0; e < 8; ++e) qs[r][e] *= scale2;
    }
    // entries that count, one lane each: above all before them and up to the own block
    int j_lane = lane < a.NS ? row[lane] : -1, high = j_lane >= 0 && j_lane <= own ? j_lane : -1;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(high, d);
        if (lane >= d) high = max(high, x);
    }
    const int before = __shfl_up(high, 1);
    const bool counts = j_lane >= 0 && j_lane <= own && (lane == 0 || j_lane > before);
    uint64_t valid = __ballot(counts);
    const int halves = a.BK / 32;
    int n = 0;                                                 // pieces of 32 keys, dealt to the wavefronts in turn
    for (; valid; valid &= valid - 1) {
        const int j = __shfl(j_lane, __ffsll((unsigned long long)valid) - 1);
        for (int half = 0; half < halves; ++half, ++n) {
            if (n % WAVES != wave) continue;
            const int key0 = j * a.BK + half * 32;
            if (key0 > p) continue;
            float ks[STEPS][8], vs[STEPS][8];
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int key = key0 + s * KEYS + key_of;
#pragma unroll
                for (int e = 0; e < 8; ++e) ks[s][e] = vs[s][e] = 0.f;
                if (mine && key <= p) {
                    load8(k.at(b, key, g) + c * 8, ks[s]);
                    load8(v.at(b, key, g) + c * 8, vs[s]);
                }
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float x[STEPS], top = -INFINITY;
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    float d = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) d += qs[r][e] * ks[s][e];
                    d = lanes_sum<LANES>(d);
                    x[s] = key0 + s * KEYS + key_of <= p ? d : -INFINITY;
                    top = fmaxf(top, x[s]);
                }
#pragma unroll
                for (int d = LANES; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
                const float to = fmaxf(m[r], top), f = exp2f(m[r] - to);     // (key0 is visible: `to` is a number)
                m[r] = to;
                l[r] *= f;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[r][e] *= f;
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const float w = exp2f(x[s] - to);
                    l[r] += w;
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[r][e] += w * vs[s][e];
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
#pragma unroll
        for (int d = LANES; d < 64; d <<= 1) {
            l[r] += __shfl_xor(l[r], d);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[r][e] += __shfl_xor(acc[r][e], d);
        }
        if (key_of == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) part[wave][r][c * 8 + e] = acc[r][e];
            if (c == 0) part_m[wave][r] = m[r], part_l[wave][r] = l[r];
        }
    }
    __syncthreads();
    for (int u = threadIdx.x; u < RT * LANES * 2; u += DEC_THREADS) {          // four components of a head to a thread
        const int r = u / (LANES * 2), d = (u - r * (LANES * 2)) * 4;
        if (r0 + r >= a.R || d >= a.D) continue;
        float top = -INFINITY, sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, part_m[w][r]);
        for (int w = 0; w < WAVES; ++w) {
            if (part_m[w][r] == -INFINITY) continue;
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

size_t partial_bytes(const AttentionArgs& a, int parts, int n) {
    return align_up((size_t)n * a.Tq * a.NS * a.R * parts * a.D * 4) + align_up((size_t)n * a.Tq * a.NS * a.R * parts * 8);
}

int parts_of(const mst_attention_shape* s) {
    const int held = s->type == MST_F32 && s->head_dim > 64 ? 32 : 64;
    return s->block <= held ? 1 : s->block / held;
}

// (batch, key head) that a launch takes
int group_of(const AttentionArgs& a, int parts) {
    const size_t one = partial_bytes(a, parts, 1);
    return (int)std::min<size_t>((size_t)a.B * a.G, std::max<size_t>(1, PARTIAL_BYTES / std::max<size_t>(one, 1)));
}

}  // namespace

size_t attention_fwd_bytes(const mst_attention_shape* s) {
    const AttentionArgs a = attention_args(s);
    return std::max<size_t>(256, partial_bytes(a, parts_of(s), group_of(a, parts_of(s))));
}

}  // namespace mst

extern "C" int mst_block_attention_fwd(const mst_attention_shape* s, const mst_heads* q, const mst_heads* k, const mst_heads* v, const void* plan_dev,
                                       const mst_heads* o, float* lse, void* ws, size_t ws_bytes, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    if (int e = check_heads(q, s->batch, s->queries, s->heads, s->type, false)) return e;
    if (int e = check_heads(k, s->batch, s->keys, s->kv_heads, s->type, false)) return e;
    if (int e = check_heads(v, s->batch, s->keys, s->kv_heads, s->type, false)) return e;
    if (int e = check_heads(o, s->batch, s->queries, s->heads, s->type, true)) return e;
    if (!plan_dev || !lse || !ws || !aligned16(plan_dev) || !aligned16(lse) || !aligned16(ws)) return MST_ERR_ARG;
    if (ws_bytes < attention_fwd_bytes(s)) return MST_ERR_WORKSPACE;
    const AttentionArgs a = attention_args(s);
    if (a.B == 0 || a.Tq == 0) return MST_OK;
    const Plan plan = carve_plan(const_cast<void*>(plan_dev), a);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int parts = parts_of(s), group = group_of(a, parts);
    const Partials part{static_cast<float*>(ws), reinterpret_cast<float2*>(static_cast<char*>(ws) + align_up((size_t)group * a.Tq * a.NS * a.R * parts * a.D * 4))};
    int status = MST_OK;
    with_type(s->type, [&](auto type) {
        using T = decltype(type);
        const Heads<const T> qh = heads_of<const T>(q), kh = heads_of<const T>(k), vh = heads_of<const T>(v);
        const Heads<T> oh = heads_of<T>(o);
        for (int bg = 0; bg < a.B * a.G && status == MST_OK; bg += group) {
            const unsigned n = (unsigned)std::min(group, a.B * a.G - bg);
            const dim3 grid((unsigned)(plan.max_items * parts), n);
            if (a.nb > 0) {
                if (a.D <= 64) {
                    if (a.BK == 32) k_attention_fwd<T, 64, 32><<<grid, FWD_THREADS, 0, st>>>(a, plan, qh, kh, vh, bg, part);
                    else k_attention_fwd<T, 64, 64><<<grid, FWD_THREADS, 0, st>>>(a, plan, qh, kh, vh, bg, part);
                } else {
                    constexpr int KW = keys_held<T, 128>();
                    if (a.BK == 32) k_attention_fwd<T, 128, 32><<<grid, FWD_THREADS, 0, st>>>(a, plan, qh, kh, vh, bg, part);
                    else k_attention_fwd<T, 128, KW><<<grid, FWD_THREADS, 0, st>>>(a, plan, qh, kh, vh, bg, part);
                }
            }
            if (a.D <= 64) k_attention_join<T, 16><<<dim3((unsigned)cdiv((int64_t)a.Tq * a.R, 16), n), 256, 0, st>>>(a, plan, parts, bg, part, oh, lse);
            else k_attention_join<T, 32><<<dim3((unsigned)cdiv((int64_t)a.Tq * a.R, 8), n), 256, 0, st>>>(a, plan, parts, bg, part, oh, lse);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) {
                g_last_hip_error = (int)e;
                status = MST_ERR_HIP;
            }
        }
    });
    return status;
}

extern "C" int mst_block_attention_decode(const mst_attention_shape* s, const mst_heads* q, const mst_heads* k, const mst_heads* v, const int32_t* blocks,
                                          const mst_heads* o, float* lse, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    if (int e = check_heads(q, s->batch, s->queries, s->heads, s->type, false)) return e;
    if (int e = check_heads(k, s->batch, s->keys, s->kv_heads, s->type, false)) return e;
    if (int e = check_heads(v, s->batch, s->keys, s->kv_heads, s->type, false)) return e;
    if (int e = check_heads(o, s->batch, s->queries, s->heads, s->type, true)) return e;
    if (!blocks || !aligned16(blocks) || !aligned16(lse)) return MST_ERR_ARG;
    const AttentionArgs a = attention_args(s);
    if (a.B == 0 || a.Tq == 0) return MST_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    with_type(s->type, [&](auto type) {
        using T = decltype(type);
        const Heads<const T> qh = heads_of<const T>(q), kh = heads_of<const T>(k), vh = heads_of<const T>(v);
        const Heads<T> oh = heads_of<T>(o);
        auto launch = [&](auto lanes, auto rt) {
            constexpr int L = decltype(lanes)::value, RT = decltype(rt)::value;
            k_attention_decode<T, L, RT><<<dim3((unsigned)(cdiv(a.R, RT) * a.Tq), (unsigned)(a.B * a.G)), DEC_THREADS, 0, st>>>(a, qh, kh, vh, blocks, oh, lse);
        };
        auto width = [&](auto rt) {
            if (a.D <= 64) launch(std::integral_constant<int, 8>{}, rt);
            else launch(std::integral_constant<int, 16>{}, rt);
        };
        if (a.R == 1) width(std::integral_constant<int, 1>{});
        else if (a.R == 2) width(std::integral_constant<int, 2>{});
        else width(std::integral_constant<int, 4>{});
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}
