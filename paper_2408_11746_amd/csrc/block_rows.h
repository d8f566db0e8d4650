// Rows (query, head) of a key head that go over their selected blocks together: what the forward and the gradient of the queries
// have in common.
//
// A workgroup owns COLS rows of consecutive queries, 32 of them a wavefront, and keeps their results in registers from the first
// block to the last.  It walks the union of the blocks that its queries selected, in ascending order: a block's keys and values
// are read once for all rows, straight to LDS, the next part of them on its way while the present one is worked on; a wavefront none of whose rows
// selected the block leaves it out, and a row that did not select it is masked.  Neighbouring queries mostly select the same
// blocks, so the union is not much more than a selection; where they do not, the work grows up to that of dense causal attention.
#pragma once

#include "block_attention.h"

namespace mst {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// Running maxima begin at the lowest number, not at -inf: scores that are -inf (products below fp32) then have the weight 2^-inf = 0, also before the first
// number, and a factor 2^(old - new) is one for an unchanged maximum.
constexpr float LOWEST = -3.402823466e38f;
constexpr int ROW_THREADS = 256, ROW_WAVES = ROW_THREADS / 64, COLS = ROW_WAVES * 32;

// Two buffers of KW keys and as many values; a load of a wavefront is 1 KB, and a wavefront moves keys or values alone
template <typename T, int DP, int KW>
struct KeyTiles {
    using R = Rows<T, DP>;
    static constexpr int TILE = KW * R::BYTES, BUFFER = 2 * TILE, BYTES = 2 * BUFFER;
    static constexpr int EACH = BUFFER / 1024 / ROW_WAVES;     // loads of a wavefront
    static_assert(EACH * ROW_WAVES * 1024 == BUFFER && TILE % (EACH * 1024) == 0, "whole loads");
    const char* base;
    int64_t stride;
    uint32_t from[EACH];                                       // byte offsets of a lane's chunks from the first key of a part
    uint32_t to;                                               // LDS address of the wavefront's first load
    int row0, last_byte;
    __device__ KeyTiles(const AttentionArgs& a, const Heads<const T>& k, const Heads<const T>& v, int b, int g, int wave, const char* lds) {
        const bool keys = wave < ROW_WAVES / 2;
        const Heads<const T>& x = keys ? k : v;
        base = reinterpret_cast<const char*>(x.at(b, 0, g));
        stride = x.st * (int64_t)sizeof(T);
        to = lds_address(lds) + wave * (EACH * 1024);
        row0 = (wave % (ROW_WAVES / 2)) * EACH * R::PER_KB;
        last_byte = a.D * (int)sizeof(T) - 16;
#pragma unroll
        for (int i = 0; i < EACH; ++i) from[i] = offset(i, KW);
    }
    // components past head_dim are read as its last ones: what they meet is zero, or is not stored
    __device__ uint32_t offset(int i, int rows) const {
        const int lane = threadIdx.x & 63, r = row0 + i * R::PER_KB + lane / R::CH;
        return (uint32_t)(min(r, rows - 1) * (int)stride + min(((lane % R::CH) ^ R::mix(r)) * 16, last_byte));
    }
    // keys key0 .. of the part to buffer `which`; keys past the sequence are read as its last one, and masked
    __device__ void load(int key0, int len, int which) const {
        const char* p = base + min(key0, len - 1) * stride;    // (a part may begin behind the last key of its block)
        const uint32_t lds = to + which * BUFFER;
        if (key0 + KW <= len) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) load_to_lds(p, from[i], lds + i * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i) load_to_lds(p, offset(i, max(len - key0, 1)), lds + i * 1024);
        }
    }
};

// LDS behind the tiles: a bit per block and wavefront, the union in order, the selections of the queries
struct UnionSpace {
    int words, list, rows, total;                              // byte offsets
    UnionSpace(const AttentionArgs& a, int tile_bytes) {
        const int tokens = COLS / a.R;
        words = tile_bytes;
        list = words + ROW_WAVES * ((a.nb + 31) / 32) * 4 + 16;                 // (its length behind the bits)
        rows = list + std::min(a.nb, tokens * a.NS) * 4;
        total = (rows + tokens * a.NS * 2 + 15) / 16 * 16;
    }
};

// grid: a workgroup per (batch, key head) and COLS / R queries.  The last queries of every head come first: theirs are the longest
// walks, and the short ones fill what they leave (8192 queries of 20 heads: forward 177 -> 142 us against head after head).
struct RowWork {
    int bg, tile;
    __device__ RowWork(int tiles) {
        const int heads = gridDim.x / tiles;
        bg = blockIdx.x % heads;
        tile = tiles - 1 - blockIdx.x / heads;
    }
};

// where a row is in its selection
struct Cursor {
    const uint16_t* row;
    int at, next;
    __device__ Cursor(const AttentionArgs& a, const uint16_t* rows, int tok, bool there) : row(rows + (there ? tok : 0) * a.NS), at(0), next(there ? rows[tok * a.NS] : a.nb) {}
    __device__ void pass(const AttentionArgs& a, int block) {  // the walk leaves `block`
        if (next == block) {
            ++at;
            next = at < a.NS ? row[at] : a.nb;
        }
    }
};

// the union of the workgroup's selections: list[i] = block | wavefronts that need it << 16.  Returns how many.
__device__ inline int make_union(const AttentionArgs& a, const int* __restrict__ selected, int t0, int tokens, uint32_t* words, uint32_t* list, uint16_t* rows) {
    const int nw = (a.nb + 31) / 32;
    int* count = reinterpret_cast<int*>(words + ROW_WAVES * nw);
    for (int i = threadIdx.x; i < ROW_WAVES * nw; i += ROW_THREADS) words[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * a.NS; i += ROW_THREADS) {
        const int tok = i / a.NS, t = t0 + tok;
        const int j = t < a.Tq ? selected[(int64_t)t0 * a.NS + i] : a.nb;
        rows[i] = (uint16_t)j;
        if (j < a.nb)
            for (int w = tok * a.R / 32; w <= (tok * a.R + a.R - 1) / 32; ++w) atomicOr(&words[w * nw + (j >> 5)], 1u << (j & 31));
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        const int w = threadIdx.x;                             // (2048 blocks: 64 words)
        uint32_t m[ROW_WAVES], all = 0;
#pragma unroll
        for (int i = 0; i < ROW_WAVES; ++i) {
            m[i] = w < nw ? words[i * nw + w] : 0u;
            all |= m[i];
        }
        int before = __popc(all), mine = before;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int x = __shfl_up(before, d);
            if (w >= d) before += x;
        }
        if (w == 63) *count = before;
        int at = before - mine;
        for (; all; all &= all - 1) {
            const int bit = __ffs(all) - 1;
            uint32_t who = 0;
#pragma unroll
            for (int i = 0; i < ROW_WAVES; ++i) who |= ((m[i] >> bit) & 1u) << i;
            list[at++] = (uint32_t)(w * 32 + bit) | who << 16;
        }
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(*count);
}

// Keys at a time: fp32 tiles are twice as large.  (64 rather than 32: 8192 queries of 20 heads of 64, forward 133 us against 148; 2 x 4099 of 24 heads of 128
// 128 against 147)
template <typename T> constexpr int keys_at_once(int block) { return sizeof(T) == 4 || block < 64 ? 32 : 64; }

}  // namespace mst
