// What the calls of the attention over selected blocks share: the shape as kernels take it, the plan and its memory.
#pragma once

#include "heads.h"

namespace mst {

struct AttentionArgs {
    int B, Tq, S, H, G, R, D;            // R query heads share a key head: H = G R
    int BK, nb, NS;                      // keys of a block, blocks of the cache, blocks of a query
    float scale;
    const int* lengths;
    __device__ int length(int b) const { return lengths ? min(max(lengths[b], 0), S) : S; }
};

// The selection as the kernels read it (a plan): the rows of blocks without the entries that do not count.  bg = b G + g.
struct Plan {
    int* rows = nullptr;                 // [bg][Tq][NS] ascending, nb behind them
    size_t total = 0;
};
inline Plan carve_plan(const void* base, const AttentionArgs& a) {
    return {static_cast<int*>(const_cast<void*>(base)), align_up(std::max<size_t>(1, (size_t)a.B * a.G * a.Tq * a.NS * 4))};
}

// The other way round, for the gradients of keys and values: the queries of each block of keys, in the workspace.  A pair is an entry of a
// query's row: query << SELECT_BITS | place.  Lists are made for `group` (batch, key head) at a time; gg counts those of a group.
constexpr int LIST_TILE = 256;           // queries that a workgroup of the builders takes
constexpr int ITEM_ROWS = 512, ITEM_ROWS_MOST = 4096;          // rows (query, head) of an item: a workgroup of the kernel that walks lists
constexpr int ITEMS = 2048;              // and about so many items, where that makes none shorter
struct Lists {
    int* list = nullptr;                 // [gg][Tq NS] pairs, block after block, ascending inside a block
    int* start = nullptr;                // [gg][nb + 1] first pair of a block
    int* item_start = nullptr;           // [gg][nb + 1] first item of a block
    int2* items = nullptr;               // [gg][max_items] block and first pair
    int* tile = nullptr;                 // [gg][tiles][nb] pairs of a block before those of this tile of queries
    int tiles = 0, max_items = 0, item_pairs = 0;
    size_t total = 0;
};

inline Lists carve_lists(void* base, const AttentionArgs& a, size_t group) {
    Lists p;
    const size_t pairs = (size_t)a.Tq * a.NS;
    const int64_t rows = (int64_t)((size_t)a.B * a.G * pairs) * a.R;
    p.tiles = (int)cdiv(a.Tq, LIST_TILE);
    p.item_pairs = (int)std::max<int64_t>(8, std::min<int64_t>(ITEM_ROWS_MOST, std::max<int64_t>(ITEM_ROWS, rows / ITEMS)) / a.R);
    p.max_items = a.nb + (int)cdiv((int64_t)pairs, p.item_pairs);
    char* c = static_cast<char*>(base);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* r = c + at;
        at = align_up(at + bytes);
        return r;
    };
    p.list = reinterpret_cast<int*>(take(group * pairs * 4));
    p.start = reinterpret_cast<int*>(take(group * (a.nb + 1) * 4));
    p.item_start = reinterpret_cast<int*>(take(group * (a.nb + 1) * 4));
    p.items = reinterpret_cast<int2*>(take(group * p.max_items * 8));
    p.tile = reinterpret_cast<int*>(take(group * p.tiles * a.nb * 4));
    p.total = at;
    return p;
}
// lists of a plan's selection for the n (batch, key head) from bg0 on (block_select.hip)
int build_lists(const AttentionArgs& a, const Plan& plan, const Lists& lists, int bg0, int n, hipStream_t s);

inline int check_attention(const mst_attention_shape* s) {
    if (!s || !is_type(s->type) || !(s->scale > -1e30f && s->scale < 1e30f) || !aligned16(s->lengths_dev)) return MST_ERR_ARG;
    if (s->batch < 0 || s->queries < 0 || s->keys < 0 || s->kv_heads < 1 || s->heads < 1 || s->heads > HEADS_MAX) return MST_ERR_SHAPE;
    if (s->heads % s->kv_heads != 0 || s->heads / s->kv_heads > 64) return MST_ERR_SHAPE;
    if (s->head_dim < 8 || s->head_dim > HEAD_DIM_MAX || s->head_dim % 8 != 0) return MST_ERR_SHAPE;
    if (s->block != 32 && s->block != 64 && s->block != 128) return MST_ERR_SHAPE;
    if (s->n_select < 1 || s->n_select > SELECT_MAX) return MST_ERR_SHAPE;
    if ((int64_t)s->keys > (int64_t)KEY_BLOCKS_MAX * s->block) return MST_ERR_SHAPE;
    // grids of (batch, key head): 65535; pairs and rows of one of them: 31 bits, as a pair itself
    if ((int64_t)s->batch * s->kv_heads > 65535) return MST_ERR_SHAPE;
    if ((int64_t)s->queries * s->n_select * (s->heads / s->kv_heads) >= (int64_t(1) << 30) || s->queries >= 1 << (31 - SELECT_BITS)) return MST_ERR_SHAPE;
    return MST_OK;
}

// keys and values go to LDS by 32-bit offsets from the first key of a part
inline int check_keys(const mst_attention_shape* s, const mst_heads* v, bool written) {
    if (int e = check_heads(v, s->batch, s->keys, s->kv_heads, s->type, written)) return e;
    return s->batch * (int64_t)s->keys > 0 && s->keys > 1 && v->token > (int64_t(1) << 22) ? MST_ERR_SHAPE : MST_OK;
}

inline AttentionArgs attention_args(const mst_attention_shape* s) {
    AttentionArgs a;
    a.B = s->batch, a.Tq = s->queries, a.S = s->keys, a.H = s->heads, a.G = s->kv_heads, a.R = s->heads / s->kv_heads, a.D = s->head_dim;
    a.BK = s->block, a.nb = (int)cdiv(s->keys, s->block), a.NS = s->n_select, a.scale = s->scale, a.lengths = s->lengths_dev;
    return a;
}

// f(T) with the storage type of the shape
template <typename F>
void with_type(mst_dtype type, F&& f) {
    if (type == MST_F32) f(float{});
    else f(bf16{});
}

}  // namespace mst
