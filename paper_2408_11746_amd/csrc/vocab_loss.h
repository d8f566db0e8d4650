// What the loss over the vocabulary keeps in its workspace, and its products (vocab_gemm.hip).
#pragma once

#include "common.h"
#include "heads.h"

namespace mst {

constexpr int VT = 256;                  // rows and columns of the largest output tile: workspace arrays are padded to it
constexpr int VK = 32;                   // contraction indices of a step
constexpr int VPAD = 64;                 // operands are padded to so many
constexpr int PLANES_MAX = 3;

// A matrix of bfloat16 numbers, or of numbers that are the sum of three (plane p a stride further on).  Along: a row's numbers are
// contraction indices; across: a row is one contraction index.  Rows past `rows` read as the last one.
struct VocabOperand {
    const uint16_t* p;
    int64_t plane, ld;
    int rows;
};

// One of the products of the loss: C[m][n] = sum_k A B
struct VocabProduct {
    VocabOperand a, b;
    const int* m_count;                  // rows of C (device), or null: m
    const int* k_count;                  // contraction indices (device), or null: k
    int m, n, k;                         // as the host knows them (the most there are)
    int planes;                          // of either operand: 1, or 3 and six products a term
    int splits;                          // of the contraction, each with its own C (sums)
    int side;                            // of a tile
};

// ---- what becomes of C
// statistics of the rows' logits, (b, sum of exp2(z log2 e - b)) per row and half a tile's columns (a wavefront's)
struct VocabStats {
    float2* stats;                       // [columns][row_stride]
    int64_t row_stride;
    int first;                           // number of the first of them
    const float* at_label;               // logit of a row's label, padded to VT
};
// the gradient of the logits d (exp(z - lse) - [label]), in planes
struct VocabLogitGrad {
    uint16_t* ds;
    int64_t plane, ld;
    const float *lse, *d;                // per row, padded to VT: infinite and 0 there
    const int* label;                    // per row, relative to the first column; the value below goes there
    const float* at_label;
    int v0;                              // of column 0 in the vocabulary
};
// fp32 sums, split s at sums + s stride; with add, added to what is there.  In blocks of 16 x 16 one after another along n, then m, padded to whole tiles: number
// 4 g + v of row r of a block is component v of its word (four numbers) 16 g + r.
struct VocabSums {
    float* sums;
    int64_t stride;
    int wide;                            // blocks along n
    int add;
};
__device__ inline int64_t sum_place(int m, int n, int wide) { return ((int64_t)(m >> 4) * wide + (n >> 4)) * 64; }      // word of the block that holds m, n
struct VocabOut {                        // rows of the result times the unit, in its type
    void* out;
    int64_t ld;
    int f32;
    const float* unit;
};

int vocab_side(int64_t m, int64_t n);    // of the tiles of a product
void vocab_splits(int m, int n, int k, int& side, int& splits);        // the same, and ranges of the contraction, for vocab_sums
// Few tokens, from the hidden states as they are: statistics per VOCAB_FEW_COLUMNS columns, [columns][tokens], and each label's logit; dz in fp32, [tokens][few_pitch(vocab)],
// and both gradients from it (either may be null), dh by way of sums [vocab_few_ranges][tokens][width]
constexpr int VOCAB_FEW_COLUMNS = 64;
__host__ __device__ constexpr int64_t few_pitch(int vocab) { return ((int64_t)vocab + VOCAB_FEW_COLUMNS - 1) / VOCAB_FEW_COLUMNS * VOCAB_FEW_COLUMNS; }
// Width 768, vocabulary 50257, forward / forward and gradients in us, this way and by tiles:
//   bf16, 16 tokens: 28 / 103 and 34 / 124; 24: - / 143 and 34 / 124.      fp32, 40: 86 / 301 and 160 / 480; 64: 117 / 405 and 160 / 480; 128: 195 / 695 and 160 / 485.
constexpr int VOCAB_FEW_BF16 = 16, VOCAB_FEW_F32 = 64;
// A small embedding is read in no time, and the launches before the tiles' count: as above, bf16, 17 tokens: width 1000, vocabulary 1200 12 / 35 and 26 / 70; width 256, vocabulary 50304 17 / 67
// and 24 / 80.
constexpr int VOCAB_FEW_SMALL = 32;
constexpr int64_t VOCAB_SMALL = int64_t(1) << 24;
inline bool vocab_is_few(const mst_vocab_loss_shape& s) {
    const int few = s.type == MST_F32 ? VOCAB_FEW_F32 : (int64_t)s.vocab * s.width <= VOCAB_SMALL ? VOCAB_FEW_SMALL : VOCAB_FEW_BF16;
    return s.tokens <= few;
}
int vocab_few(const mst_vocab_loss_shape& s, const void* h, const void* E, const int* labels, float2* stats, float* at_label, hipStream_t stream);
int vocab_few_ranges(const mst_vocab_loss_shape& s);
int vocab_few_bwd(const mst_vocab_loss_shape& s, const void* h, const void* E, const int* labels, const float* lse, const float* dloss, float* dz, float* sums, void* dh, void* dE,
                  hipStream_t stream);
int vocab_stats(const VocabProduct& p, const VocabStats& e, hipStream_t s);            // a, b along
int vocab_logit_grad(const VocabProduct& p, const VocabLogitGrad& e, hipStream_t s);   // a, b along
int vocab_sums(const VocabProduct& p, const VocabSums& e, hipStream_t s);              // a along, b across
int vocab_out(const VocabProduct& p, const VocabOut& e, hipStream_t s);                // a, b across

}  // namespace mst
