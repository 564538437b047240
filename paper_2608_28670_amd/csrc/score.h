// Attention whose scores are capped, biased by distance or masked: what its
// kernels over tensors (masked.hip) and over the 8-bit cache (kvcache.hip) share.
//
//   s(i, j) = q_i . k_j scale;  s = cap tanh(s / cap);  s -= slope_h |p_i - j|
//   o_i = sum_j e^s v_j / sum_j e^s over the keys j that query i sees, 0 if there are none
//
// Query i stands at p_i = its number + an offset.  It sees key j < n if
//   j <= p_i (causal) and |p_i - j| < window (with a window), or j < prefix;
// and if both belong to one document, where there are documents.
#pragma once

#include "attention_tile.h"

namespace bc {

// The G query heads of a key head are taken together: row r of its Tq G rows is
// query r / G of head hk G + r % G, so that all of them read its keys once.
struct ScoreArgs {
    const void *q, *k, *v;
    void* out;                              // [B, Tq, Hk G, d]
    int64_t q_batch, q_row, k_batch, k_row, v_batch, v_row;   // elements
    int B, Hk, G, Tq, Tk, d;
    const int *lens, *counts, *prefix, *q_docs, *k_docs;
    const float* slopes;
    int causal, window, q_start;
    float scale_log2;                       // scale log2(e)
    float cap_log2;                         // cap log2(e); 0: none
    float cap_exp;                          // 2 log2(e) scale / cap
    int cap_wide;                           // a cap above kCapNear: small scores take the series
    const u32x2* ranges;                    // documents of every 64 keys, [B, key tiles] (masked.hip)
    const int* order;                       // or NULL: the workgroups' rows by the tiles they visit, [B, row tiles]
    // The cache: codes of tile t of sample b and head h at ((b Hk + h) tiles + t) 128 d, scales
    // (keys, values) at the same index times two.
    const uint8_t* codes;
    const float* scales;
    int tiles;
    int parts;                              // the keys are cut into so many, joined afterwards
    float *part_o, *part_ml;                // as AttnArgs'
    int nt;                                 // keys and values past the caches
};
// tanh(z) = 1 - 2 / (1 + e^2z) is off by 2^-22 or so absolutely: with a cap c a score
// by c 2^-22, in bf16 less than a probability's own rounding up to here.
constexpr double kCapNear = 1000.0;
constexpr int kMaxPosition = 1 << 24;       // positions and their differences are exact in fp32

// How a call is laid out.
struct ScorePlan {
    int rows;       // of a workgroup: 16 (a tile a wave), 64 or 128
    int parts;
};
ScorePlan score_plan(int dtype, int B, int Hk, int64_t rows, int Tk, int d);
size_t score_part_bytes(const ScorePlan& p, int B, int Hq, int Tq, int d);

// Checks that the entry points share; each returns a status.
struct Span {
    const void* p;
    int64_t n;      // bytes
};
int score_shape(int B, int Hq, int Hk, int Tq, int Tk, int d, int dtype);
int score_options(const bc_score_opts* o, int d, ScoreArgs* a);
int score_operand(const char* name, const void* p, int64_t batch, int64_t row, int B, int64_t T, int64_t width, int dtype, Span* s);
int score_apart(const Span* written, int nw, const Span* read, int nr);      // what is written overlaps nothing else
int score_grid(const ScorePlan& p, const ScoreArgs& a);

// Joins a.parts parts into a.out.
int score_join(int dtype, const ScoreArgs& a, hipStream_t s);

}  // namespace bc
