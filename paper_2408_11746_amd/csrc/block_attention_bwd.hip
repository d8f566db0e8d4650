// Gradients of the attention over selected blocks (mst_block_attention_bwd).  With P = exp(scale q.k - lse),
// delta = sum of dO O over a row and dP = dO V^T:  dS = P (dP - delta),  dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K.
//
// Both kernels walk the plan's lists as the forward does, with the keys and values of a block in registers.  The first takes
// 32 rows at a time through LDS (Q and dO are read along the rows for S and dP and across them for dK and dV) and sums dK and
// dV in registers: no two workgroups meet in one sum, and an item leaves its sums in fp32, which a last launch adds in the order of
// the list.  The second works like the forward on S^T and leaves dQ of each (row, block).
#include "block_attention.h"

namespace mst {

size_t attention_fwd_bytes(const mst_attention_shape* s);

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int BWD_THREADS = 256, BWD_WAVES = BWD_THREADS / 64;
constexpr size_t PARTIAL_BYTES = size_t(256) << 20;

// keys that a wavefront holds: both kernels have keys, values and sums in registers
__host__ __device__ constexpr int bwd_keys(bool f32, bool wide, int block) { return f32 || wide ? 32 : (block < 64 ? block : 64); }

struct BwdArgs {
    const float* lse;                    // [B][H][Tq]
    const float* delta;                  // [B][H][Tq]
    float* dq;                           // [pair][R][parts][D]
    float* dkv;                          // [item][part][2][KW][D]
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

// what the workgroup of an item works on
struct Item {
    int bg, b, g, len, block, part, key0, first, last, index;
    bool there;
    __device__ Item(const AttentionArgs& a, const Plan& plan, int bg0, int KW) {
        bg = bg0 + blockIdx.y, b = bg / a.G, g = bg % a.G;
        const int parts = a.BK / KW;
        index = blockIdx.x / parts, part = blockIdx.x - index * parts;
        there = index < plan.item_start[(int64_t)bg * (a.nb + 1) + a.nb];
        if (!there) return;
        const int2 it = plan.items[(int64_t)bg * plan.max_items + index];
        block = it.x, first = it.y;
        last = min(first + plan.item_pairs, plan.start[(int64_t)bg * (a.nb + 1) + block + 1]);
        len = a.length(b), key0 = block * a.BK + part * KW;
    }
};

template <typename T, int DP, int KW>
__global__ __launch_bounds__(BWD_THREADS) void k_attention_dkv(AttentionArgs a, Plan plan, Heads<const T> q, Heads<const T> k, Heads<const T> v, Heads<const T> d_o,
                                                               int bg0, BwdArgs w) {
    constexpr int KT = KW / 16, DC = DP / 32, DT = DP / 16, ROW = TileRow<T, DP>::stride;
    extern __shared__ __align__(16) char lds[];
    const Item it(a, plan, bg0, KW);
    if (!it.there) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, quad = lane >> 4;
    T* qt = reinterpret_cast<T*>(lds) + wave * 2 * 32 * ROW;   // 32 rows of Q, then of dO, of this wavefront alone
    T* dt_ = qt + 32 * ROW;

    Operand<T> kf[KT][DC], vf[KT][DC];   // columns = keys
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            const int key = it.key0 + kt * 16 + i16, d = c * 32 + quad * 8;
            const bool there = key < it.len && d < a.D;
            kf[kt][c] = there ? load_operand(k.at(it.b, key, it.g) + d) : zero_operand<T>();
            vf[kt][c] = there ? load_operand(v.at(it.b, key, it.g) + d) : zero_operand<T>();
        }
    floatx4 dk[KT][DT], dv[KT][DT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int d = 0; d < DT; ++d) dk[kt][d] = dv[kt][d] = floatx4{0.f, 0.f, 0.f, 0.f};

    const int rows = (it.last - it.first) * a.R;
    const int* list = plan.list + (int64_t)it.bg * a.Tq * a.NS;
    const float scale2 = a.scale * LOG2E;
    for (int r0 = wave * 32; r0 < rows; r0 += BWD_WAVES * 32) {
        // lane l knows row l % 32: its query, log-sum, delta and the last key that it sees of this part (-1 behind the rows)
        const int row = r0 + (lane & 31);
        const bool there = row < rows;
        const int e = there ? row / a.R : 0, h = there ? row - e * a.R : 0, t = list[it.first + e] / a.NS;
        const int64_t stat = ((int64_t)it.b * a.H + it.g * a.R + h) * a.Tq + t;
        const float lse2 = there ? w.lse[stat] * LOG2E : 0.f, delta = there ? w.delta[stat] : 0.f;
        const int limit = there ? it.len - a.Tq + t - it.key0 : -1;
        const int at = there ? t * a.R + h : -1;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u0 = 0; u0 < 32 * (DP / 8); u0 += 64) {
            const int u = u0 + lane, r = u / (DP / 8), d = (u % (DP / 8)) * 8;
            const int th = __shfl(at, r);
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (th >= 0 && d < a.D) {
                const int tt = th / a.R, hh = th - tt * a.R;
                load8(q.at(it.b, tt, it.g * a.R + hh) + d, x);
                load8(d_o.at(it.b, tt, it.g * a.R + hh) + d, y);
            }
            store8(&qt[r * ROW + d], x);
            store8(&dt_[r * ROW + d], y);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        float lse_r[2][4], delta_r[2][4];
        int limit_r[2][4];
#pragma unroll
        for (int rt = 0; rt < 2; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                lse_r[rt][r] = __shfl(lse2, rt * 16 + 4 * quad + r);
                delta_r[rt][r] = __shfl(delta, rt * 16 + 4 * quad + r);
                limit_r[rt][r] = __shfl(limit, rt * 16 + 4 * quad + r);
            }
        Operand<T> pf[KT], sf[KT];       // P and dS, rows = keys, contraction over the 32 rows
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            float p[8], ds[8];
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) {
                floatx4 s = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < DC; ++c) {
                    s = product(load_operand(&qt[(rt * 16 + i16) * ROW + c * 32 + quad * 8]), kf[kt][c], s);
                    dp = product(load_operand(&dt_[(rt * 16 + i16) * ROW + c * 32 + quad * 8]), vf[kt][c], dp);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = kt * 16 + i16 <= limit_r[rt][r] ? exp2f(s[r] * scale2 - lse_r[rt][r]) : 0.f;
                    p[rt * 4 + r] = x;
                    ds[rt * 4 + r] = x * (dp[r] - delta_r[rt][r]);
                }
            }
            set_operand(pf[kt], p);
            set_operand(sf[kt], ds);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const Operand<T> qc = across<ROW>(qt + d * 16, lane), oc = across<ROW>(dt_ + d * 16, lane);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                dv[kt][d] = product(pf[kt], oc, dv[kt][d]);
                dk[kt][d] = product(sf[kt], qc, dk[kt][d]);
            }
        }
    }
    // the wavefronts' sums, one wavefront after the other: rows = keys 4 quad + r, columns = components
    float* sums = reinterpret_cast<float*>(lds);               // [2][KW][DP]
    for (int turn = 0; turn < BWD_WAVES; ++turn) {
        __syncthreads();
        if (wave != turn) continue;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float* p = &sums[(kt * 16 + 4 * quad + r) * DP + d * 16 + i16];
                    if (turn == 0) p[0] = dk[kt][d][r], p[KW * DP] = dv[kt][d][r];
                    else p[0] += dk[kt][d][r], p[KW * DP] += dv[kt][d][r];
                }
    }
    __syncthreads();
    const int parts = a.BK / KW;
    float* out = w.dkv + (((int64_t)blockIdx.y * plan.max_items + it.index) * parts + it.part) * 2 * KW * a.D;
    for (int u = threadIdx.x; u < 2 * KW * (a.D / 4); u += BWD_THREADS) {
        const int r = u / (a.D / 4), d = (u - r * (a.D / 4)) * 4;
        *reinterpret_cast<float4*>(out + r * a.D + d) = *reinterpret_cast<const float4*>(&sums[r * DP + d]);
    }
}

// dK and dV of four components of a key: the items of its block, in order
template <typename T>
__global__ __launch_bounds__(256) void k_attention_dkv_join(AttentionArgs a, Plan plan, int KW, int bg0, BwdArgs w, Heads<T> dk, Heads<T> dv) {
    const int bg = bg0 + blockIdx.y, b = bg / a.G, g = bg % a.G, units = a.D / 4, parts = a.BK / KW;
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t key = u / units;
    if (key >= a.S) return;
    const int d = (int)(u - key * units) * 4, block = (int)(key / a.BK), in = (int)(key - (int64_t)block * a.BK), part = in / KW;
    const int i0 = plan.item_start[(int64_t)bg * (a.nb + 1) + block], i1 = plan.item_start[(int64_t)bg * (a.nb + 1) + block + 1];
    float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = i0; i < i1; ++i) {
        const float* p = w.dkv + ((((int64_t)blockIdx.y * plan.max_items + i) * parts + part) * 2 * KW + (in - part * KW)) * a.D + d;
        const float4 s = *reinterpret_cast<const float4*>(p), z = *reinterpret_cast<const float4*>(p + (int64_t)KW * a.D);
        x[0] += s.x; x[1] += s.y; x[2] += s.z; x[3] += s.w;
        y[0] += z.x; y[1] += z.y; y[2] += z.z; y[3] += z.w;
    }
    store4(dk.at(b, key, g) + d, x[0] * a.scale, x[1] * a.scale, x[2] * a.scale, x[3] * a.scale);
    store4(dv.at(b, key, g) + d, y[0], y[1], y[2], y[3]);
}

template <typename T, int DP, int KW>
__global__ __launch_bounds__(BWD_THREADS) void k_attention_dq(AttentionArgs a, Plan plan, Heads<const T> q, Heads<const T> k, Heads<const T> v, Heads<const T> d_o,
                                                              int bg0, BwdArgs w) {
    constexpr int KT = KW / 16, DC = DP / 32, DT = DP / 16, KS = KW / 32, ROW = TileRow<T, DP>::stride;
    __shared__ __align__(16) T kt_[KW * ROW];
    const Item it(a, plan, bg0, KW);
    if (!it.there) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, quad = lane >> 4, parts = a.BK / KW;
    Operand<T> kf[KT][DC], vf[KT][DC], kc[DT][KS];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            const int key = it.key0 + kt * 16 + i16, d = c * 32 + quad * 8;
            const bool there = key < it.len && d < a.D;
            kf[kt][c] = there ? load_operand(k.at(it.b, key, it.g) + d) : zero_operand<T>();
            vf[kt][c] = there ? load_operand(v.at(it.b, key, it.g) + d) : zero_operand<T>();
        }
    for (int u = threadIdx.x; u < KW * (DP / 8); u += BWD_THREADS) {
        const int r = u / (DP / 8), d = (u % (DP / 8)) * 8;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (it.key0 + r < it.len && d < a.D) load8(k.at(it.b, it.key0 + r, it.g) + d, x);
        store8(&kt_[r * ROW + d], x);
    }
    __syncthreads();
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int s = 0; s < KS; ++s) kc[dt][s] = across<ROW>(&kt_[s * 32 * ROW + dt * 16], lane);

    const int rows = (it.last - it.first) * a.R;
    const int* list = plan.list + (int64_t)it.bg * a.Tq * a.NS;
    const int64_t pair0 = (int64_t)blockIdx.y * a.Tq * a.NS;
    const float scale2 = a.scale * LOG2E;
    for (int r0 = wave * 16; r0 < rows; r0 += BWD_WAVES * 16) {
        const int row = r0 + i16;
        const bool there = row < rows;
        const int e = there ? row / a.R : 0, h = there ? row - e * a.R : 0;
        const int pair = list[it.first + e], t = pair / a.NS;
        const int64_t stat = ((int64_t)it.b * a.H + it.g * a.R + h) * a.Tq + t;
        const float lse2 = w.lse[stat] * LOG2E, delta = w.delta[stat];
        const T *qp = q.at(it.b, t, it.g * a.R + h), *op = d_o.at(it.b, t, it.g * a.R + h);
        Operand<T> qf[DC], of[DC];
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            const int d = c * 32 + quad * 8;
            qf[c] = d < a.D ? load_operand(qp + d) : zero_operand<T>();
            of[c] = d < a.D ? load_operand(op + d) : zero_operand<T>();
        }
        const int limit = it.len - a.Tq + t - it.key0;
        Operand<T> sf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            float ds[8];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int kt = 2 * ks + half;
                floatx4 s = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < DC; ++c) {
                    s = product(kf[kt][c], qf[c], s);
                    dp = product(vf[kt][c], of[c], dp);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    ds[half * 4 + r] = kt * 16 + 4 * quad + r <= limit ? exp2f(s[r] * scale2 - lse2) * (dp[r] - delta) : 0.f;
            }
            set_operand(sf[ks], ds);
        }
        float* out = w.dq + (((pair0 + pair) * a.R + h) * parts + it.part) * a.D;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) x = product(kc[dt][ks], sf[ks], x);
            const int d = dt * 16 + 4 * quad;
            if (there && d < a.D) store4(out + d, x[0], x[1], x[2], x[3]);
        }
    }
}

template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_attention_dq_join(AttentionArgs a, Plan plan, int parts, int bg0, BwdArgs w, Heads<T> dq) {
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (row >= (int64_t)a.Tq * a.R || lane * 4 >= a.D) return;
    const int t = (int)(row / a.R), h = (int)(row - (int64_t)t * a.R), bg = bg0 + blockIdx.y, b = bg / a.G, g = bg % a.G;
    const int64_t pair0 = (int64_t)blockIdx.y * a.Tq * a.NS + (int64_t)t * a.NS;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    for (uint64_t v = plan.valid[(int64_t)bg * a.Tq + t]; v; v &= v - 1) {
        const float* p = w.dq + ((pair0 + __ffsll((unsigned long long)v) - 1) * a.R + h) * parts * a.D + lane * 4;
        for (int i = 0; i < parts; ++i) {
            const float4 y = *reinterpret_cast<const float4*>(p + (int64_t)i * a.D);
            x[0] += y.x; x[1] += y.y; x[2] += y.z; x[3] += y.w;
        }
    }
    store4(dq.at(b, t, g * a.R + h) + lane * 4, x[0] * a.scale, x[1] * a.scale, x[2] * a.scale, x[3] * a.scale);
}

struct BwdSpace {
    int KW, parts, group, max_items;
    size_t delta, dq, total;
};

BwdSpace bwd_space(const mst_attention_shape* s) {
    const AttentionArgs a = attention_args(s);
    BwdSpace w;
    w.KW = bwd_keys(s->type == MST_F32, s->head_dim > 64, s->block);
    w.parts = a.BK / w.KW;
    w.max_items = carve_plan(nullptr, a).max_items;
    w.delta = align_up((size_t)a.B * a.H * a.Tq * 4);
    const size_t dq1 = (size_t)a.Tq * a.NS * a.R * w.parts * a.D * 4, dkv1 = (size_t)w.max_items * 2 * a.BK * a.D * 4;
    w.group = (int)std::min<size_t>((size_t)a.B * a.G, std::max<size_t>(1, PARTIAL_BYTES / std::max<size_t>(dq1 + dkv1, 1)));
    w.dq = align_up(w.group * dq1);
    w.total = std::max<size_t>(256, w.delta + w.dq + align_up(w.group * dkv1));
    return w;
}

template <typename T, int DP, int KW>
int launch_bwd(const AttentionArgs& a, const Plan& plan, const BwdSpace& sp, const Heads<const T>& q, const Heads<const T>& k, const Heads<const T>& v, const Heads<const T>& d_o, const Heads<T>& dq, const Heads<T>& dk, const Heads<T>& dv, const BwdArgs& w, hipStream_t st) {
    constexpr int ROW = TileRow<T, DP>::stride;
    constexpr int tiles = BWD_WAVES * 2 * 32 * ROW * (int)sizeof(T), sums = 2 * KW * DP * 4, lds = tiles > sums ? tiles : sums;
    static_assert(lds <= 160 * 1024, "LDS of a CU");
    static uint64_t allowed = 0;
    const void* kernel = reinterpret_cast<const void*>(&k_attention_dkv<T, DP, KW>);
    if (int e = allow_lds(kernel, lds, allowed)) return e;
    for (int bg = 0; bg < a.B * a.G; bg += sp.group) {
        const unsigned n = (unsigned)std::min(sp.group, a.B * a.G - bg);
        const dim3 grid((unsigned)(plan.max_items * sp.parts), n);
        if (a.nb > 0 && a.Tq > 0) {
            k_attention_dkv<T, DP, KW><<<grid, BWD_THREADS, lds, st>>>(a, plan, q, k, v, d_o, bg, w);
            MST_LAUNCH_CHECK();
            k_attention_dq<T, DP, KW><<<grid, BWD_THREADS, 0, st>>>(a, plan, q, k, v, d_o, bg, w);
            MST_LAUNCH_CHECK();
        }
        if (a.S > 0) k_attention_dkv_join<T><<<dim3((unsigned)cdiv((int64_t)a.S * (a.D / 4), 256), n), 256, 0, st>>>(a, plan, KW, bg, w, dk, dv);
        MST_LAUNCH_CHECK();
        constexpr int L = DP / 4;
        if (a.Tq > 0) k_attention_dq_join<T, L><<<dim3((unsigned)cdiv((int64_t)a.Tq * a.R, 256 / L), n), 256, 0, st>>>(a, plan, sp.parts, bg, w, dq);
        MST_LAUNCH_CHECK();
    }
    return MST_OK;
}

}  // namespace
}  // namespace mst

extern "C" size_t mst_block_attention_workspace_bytes(const mst_attention_shape* s, int backward) {
    using namespace mst;
    if (check_attention(s)) return 0;
    const size_t f = attention_fwd_bytes(s);
    return backward ? std::max(f, bwd_space(s).total) : f;
}

extern "C" int mst_block_attention_bwd(const mst_attention_shape* s, const mst_heads* q, const mst_heads* k, const mst_heads* v, const void* plan_dev,
                                       const mst_heads* o, const float* lse, const mst_heads* d_o, const mst_heads* dq, const mst_heads* dk, const mst_heads* dv,
                                       void* ws, size_t ws_bytes, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_attention(s)) return e;
    const struct { const mst_heads* v; bool key, written; } views[] = {{q, false, false}, {k, true, false}, {v, true, false}, {o, false, false}, {d_o, false, false}, {dq, false, true}, {dk, true, true}, {dv, true, true}};
    for (const auto& x : views)
        if (int e = check_heads(x.v, s->batch, x.key ? s->keys : s->queries, x.key ? s->kv_heads : s->heads, s->type, x.written)) return e;
    if (!plan_dev || !lse || !ws || !aligned16(plan_dev) || !aligned16(lse) || !aligned16(ws)) return MST_ERR_ARG;
    const BwdSpace sp = bwd_space(s);
    if (ws_bytes < sp.total) return MST_ERR_WORKSPACE;
    const AttentionArgs a = attention_args(s);
    if (a.B == 0) return MST_OK;
    const Plan plan = carve_plan(const_cast<void*>(plan_dev), a);
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* base = static_cast<char*>(ws);
    const BwdArgs w{lse, reinterpret_cast<float*>(base), reinterpret_cast<float*>(base + sp.delta), reinterpret_cast<float*>(base + sp.delta + sp.dq)};
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
        constexpr bool f32 = sizeof(T) == 4;
        if (a.D <= 64) {
            if (a.BK == 32) status = launch_bwd<T, 64, 32>(a, plan, sp, qh, kh, vh, doh, dqh, dkh, dvh, w, st);
            else status = launch_bwd<T, 64, bwd_keys(f32, false, 64)>(a, plan, sp, qh, kh, vh, doh, dqh, dkh, dvh, w, st);
        } else {
            status = launch_bwd<T, 128, 32>(a, plan, sp, qh, kh, vh, doh, dqh, dkh, dvh, w, st);
        }
    });
    return status;
}
