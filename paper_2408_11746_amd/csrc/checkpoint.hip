// Activations in 8 bits (mst_checkpoint_write, _read) and the activation between fc1 and fc2 with its gradient (mst_gelu_fwd, _bwd), which
// writes and reads them beside its other operands: nothing but a pass over memory, and bound by that.  8192 x 5120 numbers, fp32 to bfloat16: 43 us (252 MB, 5.8 TB/s); the
// gradient from fp32 to bfloat16 72 (420 MB, 5.8 TB/s).  16384 x 4096 with the 8-bit form: 83 us (471 MB, 5.7 TB/s); the gradient from it and y again 99 (604 MB, 6.1 TB/s).
// The erf form is bound by the vector instructions of erfcf: 8192 x 5120 numbers to bfloat16 55 us from fp32 and 52 from bfloat16 (tanh, calls repeated in the same way: 38 and 29), the gradients 76 and 63 (73 and 42).
// 4096 x 768 bfloat16 numbers into 8 bits or back: 4.2 us, a launch; 4099 x 1601 in fp32 8.3 and 8.0 (33 MB).
//
// 32 lanes take a group of 128 columns, four to a lane, so that a group's largest number is found within half a wavefront.  Where rows are whole groups, or no units are
// involved, the groups of all rows are one sequence; only rows that end inside a group are looked up by division.
#include "rows.h"

namespace mst {
namespace {

constexpr int THREADS = 256;
constexpr int GROUPS_A_BLOCK = THREADS / 32;

struct Groups {
    int64_t count;               // groups
    int64_t numbers;             // rows x width
    int width, per_row;          // per_row 0: one sequence
};
// (A launch has less than 2^32 threads along x: the rest along y.)
constexpr int BLOCKS_ALONG = 1 << 22;
__device__ inline int64_t group_of_thread() { return ((int64_t)blockIdx.y * BLOCKS_ALONG + blockIdx.x) * GROUPS_A_BLOCK + (threadIdx.x >> 5); }
struct Place {
    int64_t at;                  // first number of the lane
    int n;                       // how many of its four are there (may be below 0)
};
__device__ inline Place place_of(const Groups& g, int64_t group, int lane) {
    if (g.per_row == 0) {
        const int64_t at = group * KEPT_GROUP + 4 * lane;
        return {at, (int)min<int64_t>(4, g.numbers - at)};
    }
    const int64_t row = (uint64_t)group >> 32 ? group / g.per_row : (int64_t)((uint32_t)group / (uint32_t)g.per_row);
    const int col = (int)(group - row * g.per_row) * KEPT_GROUP + 4 * lane;
    return {row * g.width + col, min(4, g.width - col)};
}
Groups groups_of(int64_t rows, int width, bool units) {
    if (!units || width % KEPT_GROUP == 0) return {cdiv(rows * width, KEPT_GROUP), rows * width, width, 0};
    const int per_row = (int)cdiv(width, KEPT_GROUP);
    return {rows * per_row, rows * width, width, per_row};
}

// ---- x Phi(x) and its derivative
constexpr float LOG2E = 1.44269504f;
// x s with s = 1 / (1 + exp(-2u)), derivative s + x s (1 - s) 2u'.  Past |x| = 30 s is 0 or 1 in fp32 and the second term 0; held there the cube stays a number.
// (Comparisons that no number fails: it stays none.)
__device__ inline void gelu_tanh(float x, float& y, float& slope) {
    const float c = x < -30.f ? -30.f : x > 30.f ? 30.f : x, q = c * c;
    constexpr float K = 0.7978845608f;                              // sqrt(2 / pi)
    const float u = c * (K + K * 0.044715f * q);
    const float s = __builtin_amdgcn_rcpf(1.f + exp2_fast(-2.f * LOG2E * u));
    y = x * s;
    slope = s + c * s * (1.f - s) * (2.f * K + 6.f * K * 0.044715f * q);
}
__device__ inline void gelu_erf(float x, float& y, float& slope) {
    const float phi = 0.5f * erfcf(-0.70710678f * x);
    const float c = x < -30.f ? -30.f : x > 30.f ? 30.f : x;
    y = x * phi;
    slope = phi + c * exp2_fast(-0.5f * LOG2E * c * c) * 0.3989422804f;      // 1 / sqrt(2 pi)
}
template <bool ERF>
__device__ inline void gelu(float x, float& y, float& slope) {
    if constexpr (ERF) gelu_erf(x, y, slope);
    else gelu_tanh(x, y, slope);
}

template <typename T>
__global__ __launch_bounds__(THREADS) void k_checkpoint_write(Groups g, const T* __restrict__ x, int8_t* __restrict__ codes, float* __restrict__ units) {
    const int lane = threadIdx.x & 31;
    const int64_t group = group_of_thread();
    if (group >= g.count) return;
    const Place p = place_of(g, group, lane);
    float v[4];
    load_columns(x + p.at, p.n, v);
    const float unit = kept_unit(v);
    store_codes(codes + p.at, p.n, v, unit);
    if (lane == 0) units[group] = unit;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void k_checkpoint_read(Groups g, const int8_t* __restrict__ codes, const float* __restrict__ units, T* __restrict__ x) {
    const int64_t group = group_of_thread();
    if (group >= g.count) return;
    const Place p = place_of(g, group, threadIdx.x & 31);
    float v[4];
    load_codes(codes + p.at, p.n, units[group], v);
    store_columns(x + p.at, p.n, v);
}

template <typename TX, typename TY, bool ERF, bool KEPT>
__global__ __launch_bounds__(THREADS) void k_gelu(Groups g, const TX* __restrict__ x, TY* __restrict__ y, int8_t* __restrict__ codes, float* __restrict__ units) {
    const int lane = threadIdx.x & 31;
    const int64_t group = group_of_thread();
    if (group >= g.count) return;
    const Place p = place_of(g, group, lane);
    float v[4], a[4], slope;
    load_columns(x + p.at, p.n, v);
    if constexpr (KEPT) {
        const float unit = kept_unit(v);
        store_codes(codes + p.at, p.n, v, unit);
        if (lane == 0) units[group] = unit;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) gelu<ERF>(v[e], a[e], slope);
    store_columns(y + p.at, p.n, a);
}

// TX int8_t: from what was kept.  (dx may be dy: a lane has read its numbers before it writes them.)
template <typename TX, typename TG, typename TD, typename TY, bool ERF>
__global__ __launch_bounds__(THREADS) void k_gelu_bwd(Groups g, const TX* __restrict__ x, const float* __restrict__ units, const TG* dy, TD* dx, TY* __restrict__ y) {
    const int64_t group = group_of_thread();
    if (group >= g.count) return;
    const Place p = place_of(g, group, threadIdx.x & 31);
    float v[4], d[4], a[4];
    load_columns(dy + p.at, p.n, d);
    if constexpr (sizeof(TX) == 1) load_codes(x + p.at, p.n, units[group], v);
    else load_columns(x + p.at, p.n, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float slope;
        gelu<ERF>(v[e], a[e], slope);
        d[e] *= slope;
    }
    store_columns(dx + p.at, p.n, d);
    if (y) store_columns(y + p.at, p.n, a);
}

int check_rows(int64_t rows, int32_t width) {
    if (rows < 0 || width < 1 || width > (1 << 24) || rows >= (int64_t(1) << 40) / width || rows * cdiv(width, KEPT_GROUP) > (int64_t(1) << 33)) return MST_ERR_SHAPE;
    return MST_OK;
}
int check_gelu(const mst_gelu_shape* s) {
    if (!s || !is_type(s->in_type) || !is_type(s->out_type) || !is_type(s->grad_type) || !is_type(s->in_grad_type)) return MST_ERR_ARG;
    return check_rows(s->rows, s->width);
}
bool given(const void* p) { return p && aligned16(p); }
dim3 blocks_of(const Groups& g) {
    const int64_t blocks = cdiv(g.count, GROUPS_A_BLOCK);
    return dim3((unsigned)std::min<int64_t>(blocks, BLOCKS_ALONG), (unsigned)cdiv(blocks, BLOCKS_ALONG));
}

// f(a number of the type)
template <typename F>
void with_type(mst_dtype t, F&& f) {
    if (t == MST_F32) f(float{});
    else f(bf16{});
}
template <typename F>
void with_form(int erf, F&& f) {
    if (erf) f(std::true_type{});
    else f(std::false_type{});
}

}  // namespace
}  // namespace mst

extern "C" int mst_checkpoint_write(int64_t rows, int32_t width, const void* x, mst_dtype type, const mst_checkpoint8* kept, mst_stream_t stream) {
    using namespace mst;
    if (!is_type(type) || !kept) return MST_ERR_ARG;
    if (int e = check_rows(rows, width)) return e;
    if (rows == 0) return MST_OK;
    if (!given(x)) return MST_ERR_ARG;
    if (int e = check_kept(kept)) return e;
    const Groups g = groups_of(rows, width, true);
    with_type(type, [&](auto t) {
        using T = decltype(t);
        k_checkpoint_write<T><<<blocks_of(g), THREADS, 0, static_cast<hipStream_t>(stream)>>>(g, static_cast<const T*>(x), kept->codes_dev, kept->units_dev);
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}

extern "C" int mst_checkpoint_read(int64_t rows, int32_t width, const mst_checkpoint8* kept, mst_dtype type, void* x, mst_stream_t stream) {
    using namespace mst;
    if (!is_type(type) || !kept) return MST_ERR_ARG;
    if (int e = check_rows(rows, width)) return e;
    if (rows == 0) return MST_OK;
    if (!given(x)) return MST_ERR_ARG;
    if (int e = check_kept(kept)) return e;
    const Groups g = groups_of(rows, width, true);
    with_type(type, [&](auto t) {
        using T = decltype(t);
        k_checkpoint_read<T><<<blocks_of(g), THREADS, 0, static_cast<hipStream_t>(stream)>>>(g, kept->codes_dev, kept->units_dev, static_cast<T*>(x));
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}

extern "C" int mst_gelu_fwd(const mst_gelu_shape* s, const void* x, void* y, const mst_checkpoint8* kept, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_gelu(s)) return e;
    if (s->rows == 0) return MST_OK;
    if (!given(x) || !given(y)) return MST_ERR_ARG;
    if (kept)
        if (int e = check_kept(kept)) return e;
    const Groups g = groups_of(s->rows, s->width, kept != nullptr);
    hipStream_t st = static_cast<hipStream_t>(stream);
    with_type(s->in_type, [&](auto tx) {
        with_type(s->out_type, [&](auto ty) {
            with_form(s->erf, [&](auto form) {
                using TX = decltype(tx);
                using TY = decltype(ty);
                constexpr bool ERF = decltype(form)::value;
                if (kept)
                    k_gelu<TX, TY, ERF, true><<<blocks_of(g), THREADS, 0, st>>>(g, static_cast<const TX*>(x), static_cast<TY*>(y), kept->codes_dev, kept->units_dev);
                else
                    k_gelu<TX, TY, ERF, false><<<blocks_of(g), THREADS, 0, st>>>(g, static_cast<const TX*>(x), static_cast<TY*>(y), nullptr, nullptr);
            });
        });
    });
    MST_LAUNCH_CHECK();
    return MST_OK;
}

extern "C" int mst_gelu_bwd(const mst_gelu_shape* s, const void* x, const mst_checkpoint8* kept, const void* dy, void* dx, void* y, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_gelu(s)) return e;
    if ((x != nullptr) == (kept != nullptr) && s->rows > 0) return MST_ERR_ARG;
    if (s->rows == 0) return MST_OK;
    if (!given(dy) || !given(dx) || !aligned16(x) || !aligned16(y)) return MST_ERR_ARG;
    if (dx == dy && s->grad_type != s->in_grad_type) return MST_ERR_ARG;
    if (kept)
        if (int e = check_kept(kept)) return e;
    const Groups g = groups_of(s->rows, s->width, kept != nullptr);
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto launch = [&](const auto* from, const float* units) {
        using TX = std::remove_cv_t<std::remove_pointer_t<decltype(from)>>;
        with_type(s->grad_type, [&](auto tg) {
            with_type(s->in_grad_type, [&](auto td) {
                with_type(s->out_type, [&](auto ty) {
                    with_form(s->erf, [&](auto form) {
                        using TG = decltype(tg);
                        using TD = decltype(td);
                        using TY = decltype(ty);
                        k_gelu_bwd<TX, TG, TD, TY, decltype(form)::value><<<blocks_of(g), THREADS, 0, st>>>(g, from, units, static_cast<const TG*>(dy), static_cast<TD*>(dx),
                                                                                                             static_cast<TY*>(y));
                    });
                });
            });
        });
    };
    if (kept) launch(static_cast<const int8_t*>(kept->codes_dev), kept->units_dev);
    else if (s->in_type == MST_F32) launch(static_cast<const float*>(x), nullptr);
    else launch(static_cast<const bf16*>(x), nullptr);
    MST_LAUNCH_CHECK();
    return MST_OK;
}
