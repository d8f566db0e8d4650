// Softmax cross entropy over the vocabulary from hidden states and embedding, and its gradients (mst_vocab_loss_fwd, _bwd).
//
//   z = h E^T,  lse = log sum_v exp z_v,  loss = lse - z_label;   dz = dloss (exp(z - lse) - [v = label]),  dh = dz E,  dE = dz^T h
// The logits never reach memory.  The forward reduces each tile of them to a sum per row; a second kernel joins those.  The backward
// forms them again, a piece of the vocabulary at a time (of PIECE_BYTES at most, or 256 columns), such that dz of a piece is read by both products behind it before the next
// piece replaces it; dE of a piece is complete, dh is summed in fp32 over the pieces.
// dz of bfloat16 numbers is rounded to bfloat16: dh and dE are off by 1.8e-3 with it and by 1.7e-3 without, their own rounding; in three parts the products behind it would take
// three times as long.
// Tokens without a label take no part: the labelled ones are packed side by side first (in order, so that sums do not depend on chance), which also
// pads their rows to whole steps of the products.  fp32 numbers are split into three bfloat16 parts on the way, those of the embedding
// a piece at a time.
// The logit of a token's own label is a dot product of its own in fp32, and so is what it adds to dz: exp(z - lse) - 1 without cancellation.
// The products bound it (vocab_gemm.hip).  What is here takes, of 8192 bfloat16 tokens of width 1280 and a vocabulary of 50257 (3520 us with the gradients): rows 16, packing 13 (both
// in either direction), join 8, dh 32; of 1024 tokens of width 768 (338 us): 5, 6, 7 and 10.
// Few tokens (vocab_is_few) go neither through the packing nor through pieces.
#include "rows.h"
#include "vocab_loss.h"

namespace mst {
namespace {

// Of dz and of the embedding's parts together.  Every piece costs its launches and a last round of tiles that is not full, and takes up the sums for dh again: with 512 MB 8192 tokens of width 1280,
// vocabulary 50257, have two pieces and take 3.56 ms, with 256 MB four and 3.68; fp32, 1531 tokens of width 648, vocabulary 32003, one and 1.29, two and 1.40.
constexpr int64_t PIECE_BYTES = int64_t(1) << 29;

// ---- which tokens have a label
constexpr int ROWS_THREADS = 1024, ROWS_EACH = 8;
// One workgroup: place[token] = its row or -1, list[row] = token, label[row], count.  In order.  Rows behind the last, up to a whole tile: label -1.
// Outputs of tokens without one: 0.  unit: the largest finite size of the rows' dloss (1 if all are 0; an infinite one is its own row's alone), or, where that is above 1, its
// significant digits, 1 to 2: in units of a large number itself rows of a small dloss would fall below fp32.
__global__ __launch_bounds__(ROWS_THREADS) void k_vocab_rows(const int* __restrict__ labels, int T, int V, int* __restrict__ count, int* __restrict__ place,
                                                             int* __restrict__ list, int* __restrict__ label, float* __restrict__ loss, float* __restrict__ lse,
                                                             const float* __restrict__ dloss, float* __restrict__ unit) {
    __shared__ int sums[ROWS_THREADS / 64];
    int top = 0;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int before = 0;                                                 // rows of the tokens before these
    for (int t0 = 0; t0 < T; t0 += ROWS_THREADS * ROWS_EACH) {
        int mine[ROWS_EACH], n = 0;
        float d[ROWS_EACH];
        const int first = t0 + tid * ROWS_EACH;
        if (first + ROWS_EACH <= T) {
#pragma unroll
            for (int e = 0; e < ROWS_EACH; e += 4) {
                const int4 x = *reinterpret_cast<const int4*>(labels + first + e);
                mine[e] = x.x, mine[e + 1] = x.y, mine[e + 2] = x.z, mine[e + 3] = x.w;
                if (!dloss) continue;
                const float4 y = *reinterpret_cast<const float4*>(dloss + first + e);
                d[e] = y.x, d[e + 1] = y.y, d[e + 2] = y.z, d[e + 3] = y.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < ROWS_EACH; ++e) {
                mine[e] = first + e < T ? labels[first + e] : -1;
                d[e] = dloss && first + e < T ? dloss[first + e] : 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < ROWS_EACH; ++e) {
            if (mine[e] < 0 || mine[e] >= V) mine[e] = -1;
            n += mine[e] >= 0;
        }
        int upto = n;                                               // of this wavefront's lanes up to this one
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        int row = before + upto - n;
        for (int w = 0; w < ROWS_THREADS / 64; ++w) {
            if (w < wave) row += sums[w];
            before += sums[w];
        }
#pragma unroll
        for (int e = 0; e < ROWS_EACH; ++e)
            if (first + e < T) {
                const bool has = mine[e] >= 0;
                place[first + e] = has ? row : -1;
                if (has) list[row] = first + e, label[row] = mine[e], ++row;
                const int size = __float_as_int(d[e]) & 0x7FFFFFFF;
                if (has && dloss && size < 0x7F800000) top = max(top, size);
                if (!has && loss) loss[first + e] = 0.f;
                if (!has && lse) lse[first + e] = 0.f;
            }
    }
    if (tid == 0) *count = before;
    if (dloss) {
        top = lanes_max<64>(top);
        __syncthreads();
        if (lane == 0) sums[wave] = top;
        __syncthreads();
        for (int w = 0; w < ROWS_THREADS / 64; ++w) top = max(top, sums[w]);
        constexpr int ONE = 0x3F800000;
        if (tid == 0) *unit = __int_as_float(top == 0 ? ONE : top < ONE ? top : ONE | (top & 0x007FFFFF));
    }
    const int end = (before + VT - 1) / VT * VT;
    for (int r = before + tid; r < end; r += ROWS_THREADS) label[r] = -1;
}

// x in bfloat16 parts, each what the ones before it left
__device__ inline void put_parts(uint16_t* to, int64_t plane, int planes, float (&x)[4]) {
    for (int p = 0; p < planes; ++p) {
        const uint32_t a = pack2(x[0], x[1]), b = pack2(x[2], x[3]);
        *reinterpret_cast<uint2*>(to + p * plane) = make_uint2(a, b);
        x[0] -= __uint_as_float(a << 16);
        x[1] -= __uint_as_float(a & 0xFFFF0000u);
        x[2] -= __uint_as_float(b << 16);
        x[3] -= __uint_as_float(b & 0xFFFF0000u);
    }
}

// What the packing of the rows leaves beside them, per row (zeros and an infinite lse behind the last, up to a whole tile).
// dz is held in units of the largest dloss, but for a power of two: where the loss is a mean, all dloss are one number, and the label's dz, by far the largest of a
// row, would be rounded to bfloat16 the same way in every row (2.5e-3 of dh and dE, 2.0e-3 in these units).  Both results are multiplied by the unit in fp32.
struct RowNumbers {
    float* at_label;                     // forward: the label's logit; backward: dz there
    float *lse, *d;                      // backward
    const float* unit;
};
// hidden states of the labelled tokens side by side, in parts, padded with zeros to `ld` columns and to whole steps of rows; a wavefront a row
template <typename T>
__global__ __launch_bounds__(256) void k_vocab_pack(const T* __restrict__ h, const T* __restrict__ E, int W, const int* __restrict__ count, const int* __restrict__ list,
                                                    const int* __restrict__ label, const float* __restrict__ lse, const float* __restrict__ dloss,
                                                    uint16_t* __restrict__ to, int64_t plane, int ld, int planes, RowNumbers out) {
    const int rows = *count, row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (row >= (rows + VT - 1) / VT * VT) return;
    const bool has = row < rows;
    const int token = has ? list[row] : 0;
    const T* const from = h + (int64_t)token * W;
    const T* const e = E + (int64_t)(has ? label[row] : 0) * W;
    float dot = 0.f;
    for (int c = 4 * lane; c < ld; c += 256) {
        float x[4], y[4];
        load_columns(from + c, has ? W - c : 0, x);
        load_columns(e + c, has ? W - c : 0, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) dot += x[i] * y[i];
        put_parts(to + (int64_t)row * ld + c, plane, planes, x);
    }
    dot = lanes_sum<64>(dot);
    if (lane) return;
    if (out.lse) {
        const float l = has ? lse[token] : INFINITY, d = has ? dloss[token] / *out.unit : 0.f;
        out.lse[row] = l;
        out.d[row] = d;
        out.at_label[row] = has ? d * expm1f(dot - l) : 0.f;
    } else {
        out.at_label[row] = dot;
    }
}

// rows of a piece of the embedding in parts, padded with zeros to `ld` columns and to whole steps of rows.  Bound by memory: 50257 x 768 fp32 numbers in 62 us (386 MB, 6.2 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void k_vocab_parts(const T* __restrict__ E, int rows, int padded, int W, uint16_t* __restrict__ to, int64_t plane, int ld, int planes) {
    const int64_t quads = (int64_t)padded * (ld / 4);
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < quads; q += (int64_t)gridDim.x * 256) {
        const int64_t r = q / (ld / 4);
        const int c = 4 * (int)(q - r * (ld / 4));
        float x[4];
        load_columns(E + r * W + c, r < rows ? W - c : 0, x);
        put_parts(to + r * ld + c, plane, planes, x);
    }
}

// sums of a row joined: ROWS rows a workgroup, a share of the statistics to each of its lanes of a row.  Rows are tokens (count and list null; `vocab` says which have a
// label), or the packed ones.
constexpr int JOIN_THREADS = 1024;
template <int ROWS>
__global__ __launch_bounds__(JOIN_THREADS) void k_vocab_join(const float2* __restrict__ stats, int64_t stride, int n, int tokens, const int* __restrict__ count,
                                                             const int* __restrict__ list, const int* __restrict__ labels, int vocab, const float* __restrict__ at_label,
                                                             float* __restrict__ loss, float* __restrict__ lse) {
    constexpr int SHARES = JOIN_THREADS / ROWS;
    __shared__ float2 part[SHARES][ROWS];
    const int r = threadIdx.x % ROWS, share = threadIdx.x / ROWS, row = blockIdx.x * ROWS + r, rows = count ? *count : tokens;
    if ((int)blockIdx.x * ROWS >= rows) return;
    float top = -INFINITY, sum = 0.f;
    auto add = [&](float2 x) __attribute__((always_inline)) {
        const float m = fmaxf(top, x.x), from = m == -INFINITY ? 0.f : m;
        sum = sum * exp2_fast(top - from) + x.y * exp2_fast(x.x - from);
        top = m;
    };
    if (row < rows)
#pragma unroll 8
        for (int i = share; i < n; i += SHARES) add(stats[(int64_t)i * stride + row]);
    part[share][r] = make_float2(top, sum);
    __syncthreads();
    for (int half = SHARES / 2; half > 0; half /= 2) {
        if (share < half) {
            add(part[share + half][r]);
            part[share][r] = make_float2(top, sum);
        }
        __syncthreads();
    }
    if (share || row >= rows) return;
    // 1 / (log2 e as the products of z and it have it), in two parts: lse is rounded once, and what top takes away of the loss goes away exactly
    constexpr float HIGH = 0.6931472f, LOW = 7.3486931e-9f;
    const float log_sum = log2f(sum) * HIGH, l = fmaf(top, HIGH, fmaf(top, LOW, log_sum));
    const int token = list ? list[row] : row;
    const bool has = !labels || (labels[token] >= 0 && labels[token] < vocab);
    lse[token] = has ? l : 0.f;
    if (loss) loss[token] = has ? fmaf(top, HIGH, -at_label[row]) + fmaf(top, LOW, log_sum) : 0.f;
}

// gradients of the hidden states: sums of the splits, back to the tokens' places; a wavefront takes blocks of 16 rows and 16 columns, or a workgroup's four share one
// (128 tokens of width 768, 64 splits: 33 us with a wavefront to a block, 7 with four)
template <typename T, bool SHARE>
__global__ __launch_bounds__(256) void k_vocab_dh(const float* __restrict__ sums, int64_t stride, int wide, int splits, const int* __restrict__ count, const int* __restrict__ list,
                                                  const float* __restrict__ unit, int W, T* __restrict__ dh) {
    __shared__ float4 part[4][64];
    const int rows = *count, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.x * 16 + (lane & 15), c = 16 * (SHARE ? blockIdx.y : blockIdx.y * 4 + wave);
    if ((int)blockIdx.x * 16 >= rows || c >= W) return;             // (SHARE: all of them or none)
    const float* const from = sums + 4 * (sum_place(row, c, wide) + lane);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float4 y) __attribute__((always_inline)) { x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w); };
#pragma unroll 4
    for (int s = SHARE ? wave : 0; s < splits; s += SHARE ? 4 : 1) add(*reinterpret_cast<const float4*>(from + s * stride));
    if constexpr (SHARE) {
        part[wave][lane] = x;
        __syncthreads();
        if (wave) return;
        for (int w = 1; w < 4; ++w) add(part[w][lane]);
    }
    const int col = c + 4 * (lane >> 4);
    const float u = *unit;
    if (row < rows && col < W) store4(dh + (int64_t)list[row] * W + col, u * x.x, u * x.y, u * x.z, u * x.w);
}
// ... and those of the tokens without a label: 0; a wavefront a token
template <typename T>
__global__ __launch_bounds__(256) void k_vocab_dh_others(const int* __restrict__ place, int tokens, int W, T* __restrict__ dh) {
    const int token = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (token >= tokens || place[token] >= 0) return;
    for (int c = 4 * (threadIdx.x & 63); c < W; c += 256) store4(dh + (int64_t)token * W + c, 0.f, 0.f, 0.f, 0.f);
}

int check_shape(const mst_vocab_loss_shape* s) {
    if (!s || !is_type(s->type)) return MST_ERR_ARG;
    if (s->tokens < 0 || s->tokens > (1 << 24) || s->width < 8 || s->width > 16384 || s->width % 8 || s->vocab < 1 || s->vocab > (1 << 24)) return MST_ERR_SHAPE;
    return MST_OK;
}
bool given(const void* p) { return p && aligned16(p); }

// The workspace: where its parts begin, and how the work is cut
struct Plan {
    int planes, wide;                    // parts of a number; columns of packed rows
    int side, side_dh, side_dE;          // of the tiles of logits, and of those of the gradients
    int64_t rows;                        // of packed arrays
    bool split_E;                        // the products read the embedding from its parts
    int piece, pieces;                   // columns of the vocabulary, and how often
    int splits, sum_blocks;              // of the sums for dh; blocks along a row
    bool few;                            // tokens, of which none is packed
    int stats, stat_columns;
    size_t count, unit, place, list, label, at_label, lse, d, h, E, stat, ds, sums, bytes;

    int64_t sum_stride() const { return rows * sum_blocks * 16; }
    Plan(const mst_vocab_loss_shape& s, bool backward) {
        planes = s.type == MST_F32 ? PLANES_MAX : 1;
        wide = (int)align_up(s.width, VPAD);
        rows = (int64_t)align_up(s.tokens, VT);
        split_E = planes > 1 || wide != s.width;
        const int64_t column = 2 * planes * ((backward ? rows : 0) + (split_E ? wide : 0)), whole = (int64_t)align_up(s.vocab, VT);
        const int64_t most = column == 0 ? whole : std::min(whole, std::max<int64_t>(VT, PIECE_BYTES / column / VT * VT));
        pieces = (int)cdiv(s.vocab, most);
        piece = (int)align_up(cdiv(s.vocab, pieces), VT);
        pieces = (int)cdiv(s.vocab, piece);
        few = vocab_is_few(s);
        // Logits of fp32 numbers are rounded less by small tiles, which sum small parts for themselves.  It shows in dh where few logits share a row: vocabulary 572, width 768, 2.0e-6 by large
        // tiles, 0.9e-6 by small ones (products of fp32 numbers as they are: 1.2e-6); vocabulary 32003, width 648, 0.9e-6 by large ones (3.8e-6).
        side = planes > 1 && s.vocab <= 2048 ? VT / 2 : vocab_side(s.tokens, std::min(piece, s.vocab));
        side_dE = vocab_side(std::min(piece, s.vocab), s.width);
        stat_columns = few ? VOCAB_FEW_COLUMNS : side / 2;
        stats = (int)cdiv(s.vocab, stat_columns);
        sum_blocks = (int)align_up(s.width, VT) / 16;
        side_dh = VT, splits = 1;
        if (backward && !few) vocab_splits(s.tokens, s.width, std::min(piece, s.vocab), side_dh, splits);
        bytes = 0;
        auto part = [&](size_t n) { const size_t at = bytes; bytes += align_up(n); return at; };
        if (few) {
            at_label = part(backward ? 0 : 4 * (size_t)s.tokens);
            stat = part(backward ? 0 : 8 * (size_t)s.tokens * stats);
            ds = part(backward ? 4 * (size_t)s.tokens * few_pitch(s.vocab) : 0);
            sums = part(backward ? 4 * (size_t)vocab_few_ranges(s) * s.tokens * s.width : 0);
            return;
        }
        count = part(4);
        unit = part(4);
        place = part(4 * (size_t)rows);
        list = part(4 * (size_t)rows);
        label = part(4 * (size_t)rows);
        at_label = part(4 * (size_t)rows);
        lse = part(backward ? 4 * (size_t)rows : 0);
        d = part(backward ? 4 * (size_t)rows : 0);
        h = part(2 * planes * (size_t)rows * wide);
        E = part(split_E ? 2 * planes * (size_t)piece * wide : 0);
        stat = part(backward ? 0 : 8 * (size_t)rows * stats);
        ds = part(backward ? 2 * planes * (size_t)rows * piece : 0);
        sums = part(backward ? 4 * (size_t)splits * sum_stride() : 0);
    }
};

template <typename T>
struct Run {
    const mst_vocab_loss_shape& s;
    const Plan plan;
    char* const ws;
    hipStream_t stream;
    const T *h, *E;

    template <typename N> N* at(size_t offset) const { return reinterpret_cast<N*>(ws + offset); }

    int rows(const int* labels, float* loss, float* lse, const float* lse_in, const float* dloss) const {
        k_vocab_rows<<<1, ROWS_THREADS, 0, stream>>>(labels, s.tokens, s.vocab, at<int>(plan.count), at<int>(plan.place), at<int>(plan.list), at<int>(plan.label), loss, lse,
                                                    dloss, at<float>(plan.unit));
        MST_LAUNCH_CHECK();
        const RowNumbers out = {at<float>(plan.at_label), lse_in ? at<float>(plan.lse) : nullptr, lse_in ? at<float>(plan.d) : nullptr, at<float>(plan.unit)};
        k_vocab_pack<T><<<(unsigned)(plan.rows / 4), 256, 0, stream>>>(h, E, s.width, at<int>(plan.count), at<int>(plan.list), at<int>(plan.label), lse_in, dloss,
                                                                      at<uint16_t>(plan.h), plan.rows * plan.wide, plan.wide, plan.planes, out);
        MST_LAUNCH_CHECK();
        return MST_OK;
    }
    // columns of piece i, and the embedding's rows for it
    int columns(int i) const { return std::min(plan.piece, s.vocab - i * plan.piece); }
    int embedding(int i, VocabOperand& o) const {
        const T* const from = E + (int64_t)i * plan.piece * s.width;
        const int n = columns(i);
        if (!plan.split_E) {
            o = {reinterpret_cast<const uint16_t*>(from), 0, s.width, n};
            return MST_OK;
        }
        const int padded = (int)align_up(n, VPAD);
        const int64_t quads = (int64_t)padded * (plan.wide / 4), plane = (int64_t)plan.piece * plan.wide;
        k_vocab_parts<T><<<(unsigned)std::min<int64_t>(cdiv(quads, 256), 4096), 256, 0, stream>>>(from, n, padded, s.width, at<uint16_t>(plan.E), plane, plan.wide, plan.planes);
        MST_LAUNCH_CHECK();
        o = {at<uint16_t>(plan.E), plane, plan.wide, padded};
        return MST_OK;
    }
    VocabOperand packed() const { return {at<uint16_t>(plan.h), plan.rows * plan.wide, plan.wide, (int)plan.rows}; }

    int forward(const int* labels, float* loss, float* lse) const {
        if (plan.few) {
            if (int e = vocab_few(s, h, E, labels, at<float2>(plan.stat), at<float>(plan.at_label), stream)) return e;
            return join(labels, s.tokens, loss, lse);
        }
        if (int e = rows(labels, loss, lse, nullptr, nullptr)) return e;
        for (int i = 0; i < plan.pieces; ++i) {
            VocabOperand e;
            if (int rc = embedding(i, e)) return rc;
            const VocabProduct p = {packed(), e, at<int>(plan.count), nullptr, s.tokens, columns(i), plan.wide, plan.planes, 1, plan.side};
            if (int rc = vocab_stats(p, {at<float2>(plan.stat), plan.rows, i * (plan.piece / plan.stat_columns), at<float>(plan.at_label)}, stream)) return rc;
        }
        return join(nullptr, plan.rows, loss, lse);
    }
    int join(const int* labels, int64_t stride, float* loss, float* lse) const {
        const auto kernel = plan.few ? k_vocab_join<8> : k_vocab_join<64>;
        kernel<<<(unsigned)cdiv(s.tokens, plan.few ? 8 : 64), JOIN_THREADS, 0, stream>>>(at<float2>(plan.stat), stride, plan.stats, s.tokens, labels ? nullptr : at<int>(plan.count),
                                                                                        labels ? nullptr : at<int>(plan.list), labels, s.vocab, at<float>(plan.at_label), loss, lse);
        MST_LAUNCH_CHECK();
        return MST_OK;
    }

    int backward(const int* labels, const float* lse, const float* dloss, T* dh, T* dE) const {
        if (plan.few) return vocab_few_bwd(s, h, E, labels, lse, dloss, at<float>(plan.ds), at<float>(plan.sums), dh, dE, stream);
        if (int e = rows(labels, nullptr, nullptr, lse, dloss)) return e;
        const int64_t plane = plan.rows * plan.piece;
        const VocabOperand ds_rows = {at<uint16_t>(plan.ds), plane, plan.piece, (int)plan.rows};
        for (int i = 0; i < plan.pieces; ++i) {
            const int n = columns(i);
            VocabOperand e;
            if (int rc = embedding(i, e)) return rc;
            const VocabProduct z = {packed(), e, at<int>(plan.count), nullptr, s.tokens, n, plan.wide, plan.planes, 1, plan.side};
            if (int rc = vocab_logit_grad(z, {at<uint16_t>(plan.ds), plane, plan.piece, at<float>(plan.lse), at<float>(plan.d), at<int>(plan.label), at<float>(plan.at_label),
                                             i * plan.piece}, stream)) return rc;
            if (dh) {
                const VocabProduct p = {ds_rows, e, at<int>(plan.count), nullptr, s.tokens, s.width, n, plan.planes, (int)std::min<int64_t>(plan.splits, cdiv(n, VPAD)), plan.side_dh};      // (a last piece may be short)
                if (int rc = vocab_sums(p, {at<float>(plan.sums), plan.sum_stride(), plan.sum_blocks, i > 0}, stream)) return rc;
            }
            if (dE) {
                const VocabProduct p = {ds_rows, packed(), nullptr, at<int>(plan.count), n, s.width, s.tokens, plan.planes, 1, plan.side_dE};
                if (int rc = vocab_out(p, {dE + (int64_t)i * plan.piece * s.width, s.width, s.type == MST_F32, at<float>(plan.unit)}, stream)) return rc;
            }
        }
        if (dh) {
            const bool share = plan.splits > 8;
            const auto kernel = share ? k_vocab_dh<T, true> : k_vocab_dh<T, false>;
            kernel<<<dim3((unsigned)cdiv(s.tokens, 16), (unsigned)cdiv(s.width, share ? 16 : 64)), 256, 0, stream>>>(
                at<float>(plan.sums), plan.sum_stride(), plan.sum_blocks, plan.splits, at<int>(plan.count), at<int>(plan.list), at<float>(plan.unit), s.width, dh);
            MST_LAUNCH_CHECK();
            k_vocab_dh_others<T><<<(unsigned)cdiv(s.tokens, 4), 256, 0, stream>>>(at<int>(plan.place), s.tokens, s.width, dh);
            MST_LAUNCH_CHECK();
        }
        return MST_OK;
    }
};

// dE of a batch without tokens
__global__ __launch_bounds__(256) void k_zero(uint4* __restrict__ to, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = make_uint4(0, 0, 0, 0);
}

}  // namespace
}  // namespace mst

extern "C" size_t mst_vocab_loss_workspace_bytes(const mst_vocab_loss_shape* s, int backward) {
    using namespace mst;
    if (check_shape(s)) return 0;
    const size_t forward = Plan(*s, false).bytes;
    return backward ? std::max(forward, Plan(*s, true).bytes) : forward;
}

extern "C" int mst_vocab_loss_fwd(const mst_vocab_loss_shape* s, const void* h, const void* E, const int32_t* labels, float* loss, float* lse, void* ws, size_t ws_bytes,
                                  mst_stream_t stream) {
    using namespace mst;
    if (int e = check_shape(s)) return e;
    if (s->tokens == 0) return MST_OK;
    if (!given(h) || !given(E) || !given(labels) || !given(lse) || !given(ws) || !aligned16(loss)) return MST_ERR_ARG;
    const Plan plan(*s, false);
    if (ws_bytes < plan.bytes) return MST_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (s->type == MST_F32)
        return Run<float>{*s, plan, static_cast<char*>(ws), st, static_cast<const float*>(h), static_cast<const float*>(E)}.forward(labels, loss, lse);
    return Run<bf16>{*s, plan, static_cast<char*>(ws), st, static_cast<const bf16*>(h), static_cast<const bf16*>(E)}.forward(labels, loss, lse);
}

extern "C" int mst_vocab_loss_bwd(const mst_vocab_loss_shape* s, const void* h, const void* E, const int32_t* labels, const float* lse, const float* dloss, void* dh, void* dE,
                                  void* ws, size_t ws_bytes, mst_stream_t stream) {
    using namespace mst;
    if (int e = check_shape(s)) return e;
    if (!aligned16(dh) || !aligned16(dE)) return MST_ERR_ARG;
    if (!dh && !dE) return MST_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (s->tokens == 0) {
        if (!dE) return MST_OK;
        const int64_t n = (int64_t)s->vocab * s->width * (s->type == MST_F32 ? 4 : 2) / 16;
        k_zero<<<(unsigned)std::min<int64_t>(cdiv(n, 256), 4096), 256, 0, st>>>(static_cast<uint4*>(dE), n);
        MST_LAUNCH_CHECK();
        return MST_OK;
    }
    if (!given(h) || !given(E) || !given(labels) || !given(lse) || !given(dloss) || !given(ws)) return MST_ERR_ARG;
    const Plan plan(*s, true);
    if (ws_bytes < plan.bytes) return MST_ERR_WORKSPACE;
    if (s->type == MST_F32)
        return Run<float>{*s, plan, static_cast<char*>(ws), st, static_cast<const float*>(h), static_cast<const float*>(E)}.backward(
            labels, lse, dloss, static_cast<float*>(dh), static_cast<float*>(dE));
    return Run<bf16>{*s, plan, static_cast<char*>(ws), st, static_cast<const bf16*>(h), static_cast<const bf16*>(E)}.backward(
        labels, lse, dloss, static_cast<bf16*>(dh), static_cast<bf16*>(dE));
}
