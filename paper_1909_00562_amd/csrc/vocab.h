// The operators over the vocabulary without logits: what their products' write-out needs, and the launchers of their kernels.
//
// Rows are the compacted rows of words (R of them, counted on the device), columns those of a piece of the vocabulary.
// The products leave no logits: the forward one the softmax statistics of each row's part of a tile, the logit of the
// row's word and those of its teacher entries; the backward one the derivative dl as two or three bf16 planes and its column sums.
//
// Teacher entries are kept in lists: rows in groups of 16, columns in strips of 64, the entries of a group ordered by strip, so
// that a tile finds those of its rows and columns as one run per group.  An entry is (column << 4 | row of the group) and its
// probability, that of all entries of the row with this id.
#pragma once
#include "gemm.h"

namespace asx {

constexpr int kVocabGroup = 16, kVocabStrip = 64;   // rows and columns of the lists of teacher entries
constexpr int kTeacherMaxK = 256;

struct VocabEpi {
  int32_t v0;                 // first column of the product in the vocabulary
  const int32_t* y;           // [R] word of each row
  const void* bias;           // of the product's columns, or null
  int32_t bias_f32;           // float or bf16
  float inv_tau;
  // statistics: [64 columns][ldr] each
  float2* stat;               // maximum, sum of exp relative to it
  float* stat_tau;            // teacher: sum of exp((l - maximum) / tau)
  int32_t* stat_idx;          // lowest column that attains the maximum (INT_MAX: none), or null
  int64_t ldr;
  float* at_word;             // [R]
  // teacher entries
  const int32_t* runs;        // [group][strips + 1]: a strip's first entry
  const uint32_t* ent;
  const float* ent_p;
  float* ent_l;               // out (statistics): an entry's logit
  int32_t strips;             // of the whole vocabulary
  // gradient
  const float* lse;           // [R]
  const float* lse_tau;       // [R], +inf where a row has no entries
  float a1, a2;               // dl / alpha = a1 (q - onehot) + a2 (q at temperature - p); without a teacher a1 is 1
  uint16_t* dl;               // planes of [R, ldd]
  int64_t ldd, plane;
  float* col_sums;            // [tile row][ld_sums], or null
  int64_t ld_sums;
};

constexpr int kVocabStatCols = 64;                                             // columns of a part of a row's statistics
inline int vocab_sum_rows(GemmTile t) { return t == kTile256 ? 128 : 64; }     // rows of a part of the column sums
constexpr int kVocabRowPad = 256;   // y, lse, lse_tau are read in whole tiles: their allocations are multiples of this

// terms: planes of dl (2 or 3), or 0: statistics; arg: stat_idx is wanted.  g: A, B contiguous, M_dev, no split, no C.
hipError_t launch_gemm_vocab(const GemmArgs& g, GemmTile tile, const VocabEpi& e, int terms, bool teacher, bool arg, hipStream_t st);

// ---- rows of words -------------------------------------------------------------------
struct VocabRows {
  const void* h;              // [N, H]
  bool f32;
  const int32_t* targets;
  int N, H, V, pad_id;
  int32_t *row_pos, *rows, *y, *n_act;   // y[r]: word of row r
  uint16_t* hc;               // terms of the rows of words, [plane][N, ldH]
  int64_t ldH, plane;
  float *tok_loss, *tok_distill;         // optional: 0 at padding
  int32_t* argmax;            // optional: pad_id at padding
  int32_t* ticket;            // cleared
  int32_t* chunk_words;       // words of every kRowsChunk positions, or null: not more than kRowsDirect of them
};
constexpr int kRowsChunk = 8192, kRowsDirect = 32768;
hipError_t launch_vocab_rows(const VocabRows& p, hipStream_t st);
// float [rows, H] -> three bf16 planes of [rows, ldH], zeros behind column H
hipError_t launch_vocab_terms(const float* src, int rows, int H, uint16_t* dst, int64_t ldH, int64_t plane, hipStream_t st);

// ---- few rows: the list of words' rows and the statistics in one launch, a part per kVocabFewCols words; with a teacher, whose lists want
// the rows of words first, the statistics ----
constexpr int kVocabFewCols = 128;
bool vocab_few_rows(int N, int H, bool f32, bool teacher);
hipError_t launch_vocab_few(const VocabRows& p, const VocabEpi& e, const void* W, bool arg, bool teacher, hipStream_t st);

// Backward for a few rows, both gradients in one pass over W.  epi: y, bias, lse, a1 = grad_scale, a2 = teacher's scale * tau and what
// there is of a teacher; dh_part: vocab_few_bwd_bytes.
struct VocabFewBwd {
  bool f32, g_bf16, teacher;
  const uint16_t* hc;
  int64_t ldH, plane;
  const int32_t *n_act, *row_pos;
  int N, H, V;
  const void* W;
  VocabEpi epi;
  void *dh, *dW, *db;
  float* dh_part;
};
bool vocab_few_bwd_rows(int N, int H, int V, bool f32, bool g_bf16);
size_t vocab_few_bwd_bytes(int N, int H, int V);
hipError_t launch_vocab_few_bwd(const VocabFewBwd& p, hipStream_t st);

// ---- teacher -------------------------------------------------------------------------
struct VocabTeacher {
  const int32_t* ids;         // [N, K]
  const float* logits;
  int N, K, V;
  float inv_tau;
  const int32_t *rows, *n_act;
  int32_t* runs;
  uint32_t* ent;              // [group][16 K]
  float* ent_p;
  int32_t* place;             // [R, K]: entry's index in ent, -1: none
  float* p_log_p;             // [R]: sum of p log p, 0 without entries; seen[r] says whether there are any
  int32_t* seen;
  int32_t strips;
};
hipError_t launch_vocab_teacher(const VocabTeacher& p, hipStream_t st);

// ---- joining the statistics ------------------------------------------------------------
struct VocabFinish {
  const float2* stat;
  const float* stat_tau;      // teacher, or null
  const int32_t* stat_idx;    // or null
  int64_t ldr;
  int parts;                  // tile columns of this piece
  bool first, last;           // of the pieces
  float4* run;                // [N] maximum, sum, sum at temperature, (bits) index so far: pieces in between
  const float* at_word;
  const int32_t *rows, *n_act;
  int N;
  float *lse, *lse_tau, *loss_ws, *distill_ws;
  float *tok_loss, *tok_distill;
  int32_t* argmax;
  float *loss_sum, *distill_sum;
  int32_t *n_tok, *ticket;
  // teacher
  int K;
  float inv_tau, tau2;
  const int32_t *place, *seen;
  const float *ent_p, *ent_l, *p_log_p;
};
hipError_t launch_vocab_finish(const VocabFinish& p, hipStream_t st);

// ---- gradients on their way out ----------------------------------------------------------
// dh[n] = alpha src[row_pos[n]], zeros at padding; db[v] = alpha times the column sums' parts, in order (db: optional)
struct VocabOutGrads {
  const float* src;
  const int32_t* row_pos;
  int N, H;
  int64_t ld;
  void* dh;
  const float* sums;          // [parts of sum_rows rows of words][ld_sums]
  int64_t ld_sums;
  int sum_rows;
  const int32_t* n_act;
  int V;
  void* db;
  float alpha;
};
hipError_t launch_vocab_out_grads(const VocabOutGrads& p, bool bf16, hipStream_t st);

}  // namespace asx
