// Sum of a branch and the residual stream, layer norm of it, and the gradients (mst_layer_norm_fwd, _bwd).
//
// A row stays in the registers of one wavefront (or, where it is longer than 2048 columns, of a workgroup of four or eight): every value is read once
// and written once, the mean and then the mean of the squared distances from it are sums over lanes.  Bound by memory: 8192 rows of 1280, fp32 in and bfloat16 out,
// take 25.1 us (147 MB at 5.9 TB/s); the gradients of fp32 rows 27.7 us (168 MB at 6.1 TB/s) and 4.9 for the sums of dweight and dbias; 16384 bfloat16 rows of 1024
// with their 8-bit form 28.5 us (118 MB), the gradients from that and the normed rows again 34.0 (151 MB).  32 rows of 768 take 3.7 us, a launch.
// The backward needs nothing of the forward but s: with n = (s - mean) r, r = 1 / sqrt(variance + eps) and g = dy weight,
//   dx = r (g - mean g - n mean(g n)) + ds,   dweight = sum over the rows of dy n,   dbias = sum of dy.
// A lane meets the same columns in all its rows and keeps their sums in registers; a workgroup adds its wavefronts and writes one row of sums, and
// a second launch adds those in order: the same sums in the same order every time.
#include <type_traits>

#include "rows.h"

namespace mst {
namespace {

constexpr int ROWS_A_BLOCK = 4;          // wavefronts of a workgroup whose rows are one wavefront's
constexpr int WIDTH_MAX = 16384;
constexpr int BWD_BLOCKS = 768;          // workgroups of the backward, at most (three to a CU: what its registers allow at 1280 columns): rows of the weights' sums

__host__ __device__ constexpr int pitch_of(int width) { return (width + 3) & ~3; }      // of a row of the weights' sums

struct NormRows {
    int64_t rows;
    int width;
    float eps, inverse_width;
};

// x added over the WAVES wavefronts that have a row; `room` is theirs alone until they meet again
template <int WAVES>
__device__ inline float row_sum(float x, float* room) {
    x = lanes_sum<64>(x);
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();                 // (the sums before these have been read)
        if ((threadIdx.x & 63) == 0) room[wave] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x += room[w];
    }
    return x;
}

// A lane's CH quads of a row: quad c is columns 4 (c LANES + thread) .. + 3.  A row may end in the last two of them, or in the last (ENDS).
template <int CH, int WAVES, int ENDS>
struct Span {
    static constexpr int LANES = 64 * WAVES;
    int thread, width;
    __device__ Span(int width_) : thread(WAVES == 1 ? threadIdx.x & 63 : threadIdx.x), width(width_) {}
    __device__ int column(int c) const { return 4 * (c * LANES + thread); }
    __device__ int count(int c) const { return c < CH - ENDS ? 4 : width - column(c); }          // (0 or less: none)
    // The row's address stays in scalar registers and the lane's offset is one of 32 bits: left to itself the compiler keeps a 64-bit address for each quad of each
    // operand, which take more registers than the numbers.
    template <typename T>
    __device__ void load(const T* row, float (&x)[CH][4]) const {
        auto at = (__attribute__((address_space(1))) const char*)row;
        asm("" : "+s"(at));
#pragma unroll
        for (int c = 0; c < CH; ++c) load_columns((const T*)(at + (uint32_t)(thread * 4 * (int)sizeof(T)) + c * LANES * 4 * (int)sizeof(T)), count(c), x[c]);
    }
    template <typename T>
    __device__ void store(T* row, const float (&x)[CH][4]) const {
        auto at = (__attribute__((address_space(1))) char*)row;
        asm("" : "+s"(at));
#pragma unroll
        for (int c = 0; c < CH; ++c) store_columns((T*)(at + (uint32_t)(thread * 4 * (int)sizeof(T)) + c * LANES * 4 * (int)sizeof(T)), count(c), x[c]);
    }
    // x - mean where there are columns, 0 elsewhere, and r
    __device__ float center(const NormRows& n, float (&x)[CH][4], float* room) const {
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) s += (x[c][0] + x[c][1]) + (x[c][2] + x[c][3]);
        const float mean = row_sum<WAVES>(s, room) * n.inverse_width;
        s = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[c][e] = e < count(c) ? x[c][e] - mean : 0.f;
                s += x[c][e] * x[c][e];
            }
        return 1.f / sqrtf(row_sum<WAVES>(s, room) * n.inverse_width + n.eps);
    }
};

template <int CH, int WAVES, int ENDS, typename TX, typename TY>
__global__ __launch_bounds__(64 * (WAVES == 1 ? ROWS_A_BLOCK : WAVES)) void k_layer_norm(NormRows n, const TX* x, const TX* residual, const float* __restrict__ weight,
                                                                                         const float* __restrict__ bias, TX* sum, TY* __restrict__ y,
                                                                                         int8_t* __restrict__ codes, float* __restrict__ units) {
    __shared__ float room[WAVES];
    const Span<CH, WAVES, ENDS> span(n.width);
    const int64_t first = WAVES == 1 ? (int64_t)blockIdx.x * ROWS_A_BLOCK + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x, step = (int64_t)gridDim.x * (WAVES == 1 ? ROWS_A_BLOCK : 1);
    const int per_row = (n.width + KEPT_GROUP - 1) / KEPT_GROUP;
    for (int64_t row = first; row < n.rows; row += step) {
        const int64_t at = row * n.width;
        float s[CH][4];
        span.load(x + at, s);
        if (residual) {
            float r[CH][4];
            span.load(residual + at, r);
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[c][e] += r[c][e];
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) round_columns(x, s[c]);         // what is normed is what the backward pass will find
        if (sum) span.store(sum + at, s);
        if (codes) {
            auto code_row = (__attribute__((address_space(1))) int8_t*)(codes + at);
            asm("" : "+s"(code_row));
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const float unit = kept_unit(s[c]);
                store_codes((int8_t*)(code_row + (uint32_t)(span.thread * 4) + c * span.LANES * 4), span.count(c), s[c], unit);
                const int group = span.column(c) / KEPT_GROUP;
                if ((threadIdx.x & 31) == 0 && group < per_row) units[row * per_row + group] = unit;
            }
        }
        const float r = span.center(n, s, room);
        float w[CH][4], b[CH][4];
        if (weight) span.load(weight, w);
        if (bias) span.load(bias, b);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[c][e] = s[c][e] * r * (weight ? w[c][e] : 1.f) + (bias ? b[c][e] : 0.f);
        span.store(y + at, s);
    }
}

// wavefronts of a SIMD that the registers have to suffice for
constexpr int bwd_waves(int ch, int waves) { return ch <= 3 ? 4 : waves == 1 && ch <= 5 ? 3 : 2; }
// TS int8_t: from what was kept.  (dx may be dy or ds: a row has been read before it is written.)
template <int CH, int WAVES, int ENDS, typename TS, typename TX, typename TG>
__global__ __launch_bounds__(64 * (WAVES == 1 ? ROWS_A_BLOCK : WAVES)) __attribute__((amdgpu_waves_per_eu(bwd_waves(CH, WAVES)))) void k_layer_norm_bwd(NormRows n, const TS* __restrict__ sum, const float* __restrict__ units,
                                                                                             const float* __restrict__ weight, const float* __restrict__ bias,
                                                                                             const TG* dy, const TX* ds, TX* dx, void* __restrict__ y, int y_f32,
                                                                                             float* __restrict__ partial) {
    constexpr int SHARED = WAVES == 1 ? ROWS_A_BLOCK : 1;
    __shared__ float room[WAVES];
    __shared__ float4 sums[SHARED][CH * 64 + 1];
    const Span<CH, WAVES, ENDS> span(n.width);
    const int64_t first = WAVES == 1 ? (int64_t)blockIdx.x * ROWS_A_BLOCK + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x, step = (int64_t)gridDim.x * (WAVES == 1 ? ROWS_A_BLOCK : 1);
    const int per_row = (n.width + KEPT_GROUP - 1) / KEPT_GROUP;
    float dw[CH][4], db[CH][4];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) dw[c][e] = db[c][e] = 0.f;
    for (int64_t row = first; row < n.rows; row += step) {
        const int64_t at = row * n.width;
        float s[CH][4], g[CH][4];
        if constexpr (sizeof(TS) == 1) {
            auto code_row = (__attribute__((address_space(1))) const int8_t*)(sum + at);
            auto unit_row = (__attribute__((address_space(1))) const float*)(units + row * per_row);
            asm("" : "+s"(code_row), "+s"(unit_row));
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const uint32_t group = min(span.column(c) / KEPT_GROUP, per_row - 1);
                load_codes((const int8_t*)(code_row + (uint32_t)(span.thread * 4) + c * span.LANES * 4), span.count(c), unit_row[group], s[c]);
            }
        } else {
            span.load(sum + at, s);
        }
        span.load(dy + at, g);
        const float r = span.center(n, s, room);
        float w[CH][4];                                             // (from the first cache, row by row: there are no registers for it)
        if (weight) span.load(weight, w);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) w[c][e] = weight ? w[c][e] : 1.f;
        float c1 = 0.f, c2 = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[c][e] *= r;
                dw[c][e] += g[c][e] * s[c][e];
                db[c][e] += g[c][e];
                g[c][e] *= w[c][e];
                c1 += g[c][e];
                c2 += g[c][e] * s[c][e];
            }
        c1 = row_sum<WAVES>(c1, room) * n.inverse_width;
        c2 = row_sum<WAVES>(c2, room) * n.inverse_width;
        float d[CH][4];
        if (ds) span.load(ds + at, d);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[c][e] = r * (g[c][e] - c1 - s[c][e] * c2) + (ds ? d[c][e] : 0.f);
        span.store(dx + at, d);
        if (y) {
            float b[CH][4];
            if (bias) span.load(bias, b);
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[c][e] = s[c][e] * w[c][e] + (bias ? b[c][e] : 0.f);
            if (y_f32) span.store(static_cast<float*>(y) + at, s);
            else span.store(static_cast<bf16*>(y) + at, s);
        }
    }
    if (!partial) return;
    const int pitch = pitch_of(n.width);
    float* const out = partial + (int64_t)blockIdx.x * 2 * pitch;
    auto write = [&](const float (&v)[CH][4], float* to) __attribute__((always_inline)) {
        if constexpr (WAVES == 1) {
            const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
            __syncthreads();
#pragma unroll
            for (int c = 0; c < CH; ++c) sums[wave][c * 64 + lane] = make_float4(v[c][0], v[c][1], v[c][2], v[c][3]);
            __syncthreads();
            for (int q = threadIdx.x; 4 * q < n.width; q += 64 * ROWS_A_BLOCK) {
                float4 a = sums[0][q];
#pragma unroll
                for (int o = 1; o < ROWS_A_BLOCK; ++o) {
                    const float4 b = sums[o][q];
                    a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
                }
                const float x[4] = {a.x, a.y, a.z, a.w};
                store_columns(to + 4 * q, n.width - 4 * q, x);
            }
        } else {
            span.store(to, v);
        }
    };
    write(dw, out);
    write(db, out + pitch);
}

// rows of the partial sums added: workgroup (sixteen columns, which of the two), 128 rows at a time.  7.9 MB of 768 rows of 2 x 1280 sums: 4.9 us, of which a launch is most.
__global__ __launch_bounds__(512) void k_layer_norm_sums(const float* __restrict__ partial, int width, int rows, float* __restrict__ dweight, float* __restrict__ dbias) {
    __shared__ float part[8][16];
    float* const out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int pitch = pitch_of(width), q = threadIdx.x & 3, g = threadIdx.x >> 2, col = blockIdx.x * 16 + 4 * q;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 6
    for (int r = g; r < rows; r += 128) {
        float x[4];
        load_columns(partial + ((int64_t)r * 2 + blockIdx.y) * pitch + col, width - col, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += x[e];
    }
    // over the sixteen rows of a wavefront, then the wavefronts
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int d = 4; d < 64; d *= 2) s[e] += __shfl_xor(s[e], d);
        if ((threadIdx.x & 63) < 4) part[threadIdx.x >> 6][4 * q + e] = s[e];
    }
    __syncthreads();
    const int c = threadIdx.x;
    if (c < 16 && blockIdx.x * 16 + c < width)
        out[blockIdx.x * 16 + c] = ((part[0][c] + part[1][c]) + (part[2][c] + part[3][c])) + ((part[4][c] + part[5][c]) + (part[6][c] + part[7][c]));
}

int check_shape(const mst_norm_shape* s) {
    if (!s || !is_type(s->in_type) || !is_type(s->out_type) || !is_type(s->grad_type) || !(s->eps >= 0.f) || !(s->eps <= 1e30f)) return MST_ERR_ARG;
    if (s->rows < 0 || s->rows > (int64_t(1) << 31) || s->width < 1 || s->width > WIDTH_MAX) return MST_ERR_SHAPE;
    return MST_OK;
}
bool given(const void* p) { return p && aligned16(p); }

// f(quads of a lane, wavefronts of a row, quads in which it may end).  Up to 2048 columns one wavefront has a row: no barrier, and four rows a workgroup.  Quads before the
// last are whole by the choice of their number, so that they need no checks.
template <typename F>
void with_span(int width, F&& f) {
    auto call = [&](auto ch, auto waves, auto ends) { f(ch, waves, ends); };
    std::integral_constant<int, 1> c1;
    std::integral_constant<int, 2> c2;
    std::integral_constant<int, 3> c3;
    std::integral_constant<int, 4> c4;
    std::integral_constant<int, 5> c5;
    std::integral_constant<int, 6> c6;
    std::integral_constant<int, 7> c7;
    std::integral_constant<int, 8> c8;
    switch (cdiv(width, 256)) {
        case 1: return call(c1, c1, c1);
        case 2: return call(c2, c1, c1);
        case 3: return call(c3, c1, c1);
        case 4: return call(c4, c1, c1);
        case 5: return call(c5, c1, c1);
        case 6: case 7: return call(c7, c1, c2);
        case 8: return call(c8, c1, c1);
        default: break;
    }
    if (width <= 4096) return call(c4, c4, c2);
    if (width <= 8192) return call(c4, c8, c2);
    if (width <= 12288) return call(c6, c8, c2);
    call(c8, c8, c2);
}
unsigned blocks_of(const mst_norm_shape* s, int rows_a_block, int most) { return (unsigned)std::min<int64_t>(cdiv(s->rows, s->width <= 2048 ? rows_a_block : 1), most); }

// f(numbers of the types)
template <typename F>
void with_type(mst_dtype t, F&& f) {
    if (t == MST_F32) f(float{});
    else f(bf16{});
}

}  // namespace
}  // namespace mst

extern "C" int mst_layer_norm_fwd(const mst_norm_shape* s, const void* x, const void* residual, const float* weight, const float* bias, void* sum, void* y,
                                  const mst_checkpoint8* kept, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_shape(s)) return e;
    if (s->rows == 0) return MST_OK;
    if (!given(x) || !given(y) || !aligned16(residual) || !aligned16(weight) || !aligned16(bias) || !aligned16(sum)) return MST_ERR_ARG;
    if (kept)
        if (int e = check_kept(kept)) return e;
    const NormRows n = {s->rows, s->width, s->eps, 1.f / (float)s->width};
    with_span(s->width, [&](auto ch, auto waves, auto ends) {
        with_type(s->in_type, [&](auto tx) {
            with_type(s->out_type, [&](auto ty) {
                using TX = decltype(tx);
                using TY = decltype(ty);
                constexpr int WAVES = decltype(waves)::value;
                k_layer_norm<decltype(ch)::value, WAVES, decltype(ends)::value, TX, TY><<<blocks_of(s, ROWS_A_BLOCK, 1 << 20), 64 * (WAVES == 1 ? ROWS_A_BLOCK : WAVES), 0, static_cast<hipStream_t>(stream)>>>(
                    n, static_cast<const TX*>(x), static_cast<const TX*>(residual), weight, bias, static_cast<TX*>(sum), static_cast<TY*>(y),
                    kept ? kept->codes_dev : nullptr, kept ? kept->units_dev : nullptr);
            });
        });
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}

extern "C" size_t mst_layer_norm_workspace_bytes(const mst_norm_shape* s) {
    using namespace mst;
    if (check_shape(s)) return 0;
    return align_up(std::max<size_t>(1, blocks_of(s, ROWS_A_BLOCK, BWD_BLOCKS)) * 2 * pitch_of(s->width) * sizeof(float));
}

extern "C" int mst_layer_norm_bwd(const mst_norm_shape* s, const void* sum, const mst_checkpoint8* kept, const float* weight, const float* bias, const void* dy,
                                  const void* ds, void* dx, float* dweight, float* dbias, void* y, void* ws, size_t ws_bytes, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_shape(s)) return e;
    const bool sums = dweight || dbias;
    if (!aligned16(dweight) || !aligned16(dbias) || (sums && !given(ws))) return MST_ERR_ARG;
    if (s->rows > 0) {
        if ((sum != nullptr) == (kept != nullptr)) return MST_ERR_ARG;
        if (!given(dy) || !given(dx) || !aligned16(sum) || !aligned16(ds) || !aligned16(weight) || !aligned16(bias) || !aligned16(y)) return MST_ERR_ARG;
        if (kept)
            if (int e = check_kept(kept)) return e;
    }
    if (dx == dy && dy && s->grad_type != s->in_type) return MST_ERR_ARG;
    if (sums && ws_bytes < mst_layer_norm_workspace_bytes(s)) return MST_ERR_WORKSPACE;
    const NormRows n = {s->rows, s->width, s->eps, 1.f / (float)s->width};
    const unsigned blocks = blocks_of(s, ROWS_A_BLOCK, BWD_BLOCKS);
    float* const partial = static_cast<float*>(ws);
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto launch = [&](const auto* from, const float* units, auto tx) {
        using TS = std::remove_cv_t<std::remove_pointer_t<decltype(from)>>;
        using TX = decltype(tx);
        with_span(s->width, [&](auto ch, auto waves, auto ends) {
            with_type(s->grad_type, [&](auto tg) {
                using TG = decltype(tg);
                constexpr int WAVES = decltype(waves)::value;
                k_layer_norm_bwd<decltype(ch)::value, WAVES, decltype(ends)::value, TS, TX, TG><<<blocks, 64 * (WAVES == 1 ? ROWS_A_BLOCK : WAVES), 0, st>>>(
                    n, from, units, weight, bias, static_cast<const TG*>(dy), static_cast<const TX*>(ds), static_cast<TX*>(dx), y, s->out_type == MST_F32,
                    sums ? partial : nullptr);
            });
        });
    };
    if (blocks > 0) {
        if (kept) {
            if (s->in_type == MST_F32) launch(static_cast<const int8_t*>(kept->codes_dev), kept->units_dev, float{});
            else launch(static_cast<const int8_t*>(kept->codes_dev), kept->units_dev, bf16{});
        } else if (s->in_type == MST_F32) {
            launch(static_cast<const float*>(sum), nullptr, float{});
        } else {
            launch(static_cast<const bf16*>(sum), nullptr, bf16{});
        }
        MST_LAUNCH_CHECK();
    }
    if (sums) {                           // (no rows: zeros)
        k_layer_norm_sums<<<dim3((unsigned)cdiv(s->width, 16), 2), 512, 0, st>>>(partial, s->width, (int)blocks, dweight, dbias);
        MST_LAUNCH_CHECK();
    }
    return MST_OK;
}
