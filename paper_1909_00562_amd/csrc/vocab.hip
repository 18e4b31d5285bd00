// Softmax cross-entropy over a vocabulary and distillation without keeping the logits: argument checks, workspace and the
// order of the kernels.
//
// Forward: the rows of words of h are gathered (a count that stays on the device), one product h W^T whose write-out leaves the
// softmax statistics of each row's part of a tile instead of the logits, and a pass that joins them.
// Backward, a piece of the vocabulary at a time: the product again, its write-out now dl = g (exp(l - lse) - onehot) [+ s tau
// (q - p)] and its column sums (db), then dW_piece = dl^T h and dh += dl W_piece while dl is still in the caches.
// Four products of 2 R V H where three would do with the logits kept: what that buys is R V elements of memory.
//
// dl is the sum of bf16 terms, each in a plane of its own, whose products with the other operand are reduction segments of one launch:
// three for float gradients (24 bits of mantissa), two for bf16 ones (2^-17).  One alone would be a rounding by up to 2^-8 that does not
// average out where sums cancel: sum_v dl_nv is 0, so what all rows of W have in common cancels in dh, and what the positions ask of a
// word's row cancels in dW as training goes on.  (A softmax over 4000 words x 256 fitted to 2000 positions for 20 steps: dW 0.51 % off where
// the rounding of the result makes 0.17, dh 0.31; for 60 steps 4.3 %; with two terms 0.17 throughout.)
// fp32 storage: h and W as three terms too, the six products of terms whose ranks add up to two at most; what is left out is 2^-24 of a
// product.  The planes of W are made once, or a piece at a time where all of them would take more than a piece may.
#include "../../include/vocab_ops.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "common.h"
#include "gemm.h"
#include "kernels.h"
#include "status.h"
#include "vocab.h"

namespace asx {
namespace {

constexpr size_t kAlignV = 256;
size_t upv(size_t x) { return (x + kAlignV - 1) / kAlignV * kAlignV; }
int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// What a piece of the vocabulary may take: dl of the backward pass, or the statistics or terms of W of the forward one.  Larger
// pieces fill the rounds of the compute units better, and the sums of dh are read and written once per piece; past the 256 MB of the
// memory-side cache dW and dh read dl from memory: 64 / 128 / 256 / 512 MiB, forward and backward, 2257 x 1000 x 32003 float gradients 1113 /
// 1088 / 1072 / 1161 us; bf16 gradients, 256 / 512, 2257 x 1000 x 32003 759 / 905, 5000 x 2048 x 60000 5.50 / 5.73 ms.
constexpr int64_t kPieceBytes = (int64_t)256 << 20;
constexpr int64_t kPieceColumns = 256;   // pieces are multiples of it

struct VocabLayout {
  bool f32, g_bf16;
  bool few, few_bwd;                      // few rows: a pass in one launch over W
  int h_terms, dl_terms;
  int64_t ldH, fwd_cols, bwd_cols, ldd;
  int strips, groups;
  GemmTile t_fwd, t_bwd;
  GemmPlan p_dw, p_dh;
  bool apart = false;                     // dW and dh in launches of their own
  // kept from the forward to the backward pass
  size_t rows, row_pos, chunk_words, y, n_act, ticket, hc, lse, lse_tau, at_word, loss_ws, distill_ws, run;
  size_t runs, ent, ent_p, ent_l, place, p_log_p, seen;
  // one area for the pieces of either pass
  size_t stat, stat_tau, stat_idx, w_fwd;
  bool w_kept;                            // terms of all of W, made once for both passes
  size_t dl, w_bwd, col_sums, dh_acc, partial_dw, partial_dh;
  int64_t ld_sums;
  size_t total;
};

bool types_ok(const vo_shape* s) {
  return (s->dtype == AS_F32 && s->grad_dtype == AS_F32) ||
         (s->dtype == AS_BF16 && (s->grad_dtype == AS_F32 || s->grad_dtype == AS_BF16));
}
bool shape_ok(const vo_shape* s) {
  if (s->N < 1 || s->N > (1 << 24) || s->H < 1 || s->H > (1 << 16) || s->V < 1 || s->V > (1 << 26)) return false;
  if ((int64_t)s->V * s->H >= (int64_t)1 << 40) return false;
  return s->pad_id >= -1 && s->pad_id < s->V && std::isfinite(s->grad_scale);
}
// Temperatures from 2^-10 on: a log-sum-exp of l / tau in fp32 is off by |l| / tau 2^-24, and far below that limit by so much that the
// probabilities made from it would overflow (l = 30 at tau = 1e-9: e^1800).
bool teacher_ok(const vo_shape* s, const vo_teacher* t) {
  return t->K >= 1 && t->K <= kTeacherMaxK && s->V <= (1 << 20) && round_up(s->N, kVocabGroup) * t->K < ((int64_t)1 << 31) &&
         t->temperature >= 0x1p-10f && std::isfinite(t->temperature * t->temperature) && std::isfinite(t->scale) &&
         std::isfinite(t->scale * t->temperature);
}

// pairs of terms (rank of A, rank of B), the smallest products first
int term_pairs(int a_terms, int b_terms, int (&pairs)[kMaxSeg][2]) {
  int n = 0;
  for (int sum = 2; sum >= 0; --sum)
    for (int a = 0; a <= sum; ++a)
      if (a < a_terms && sum - a < b_terms) {
        pairs[n][0] = a;
        pairs[n++][1] = sum - a;
      }
  return n;
}
int pair_count(int a_terms, int b_terms) {
  int pairs[kMaxSeg][2];
  return term_pairs(a_terms, b_terms, pairs);
}

// no split may be empty (the last piece has fewer reduction tiles than the others)
int whole_splits(int tiles, int splits) {
  if (splits > tiles) splits = tiles;
  const int per = (tiles + splits - 1) / splits;
  return (tiles + per - 1) / per;
}

int64_t piece_columns(int64_t V, int64_t bytes_per_column) {
  int64_t c = kPieceBytes / bytes_per_column / kPieceColumns * kPieceColumns;
  if (c < kPieceColumns) c = kPieceColumns;
  if (c > (1 << 20)) c = 1 << 20;
  const int64_t pieces = (V + c - 1) / c;
  return round_up((V + pieces - 1) / pieces, kPieceColumns);   // of the same size
}

// tiles of the product that makes the logits
GemmTile logits_tile(int64_t N, int64_t cols, int64_t ldH, int terms) {
  const GemmTile t = gemm_plan((int)N, (int)cols, (int)ldH * pair_count(terms, terms), 1, true, false).tile;
  // The 256 x 256 kernel's write-out runs with its matrix pipe idle, which the 128 x 128 one's second block on a compute unit hides:
  // two rounds of tiles and more are the larger kernel's.  us, forward and backward, 128 / 256: 480 words x 512 x 16000 fp32 288
  // / 396, 622 x 512 x 32003 forward 60.6 / 78.8; 1580 x 1000 x 32003 1080 / 1037, 4480 x 1024 x 32000 1264 / 1216.
  if (t == kTile64) return t;
  return ((N + 255) / 256) * ((cols + 255) / 256) >= 512 ? kTile256 : kTile128;
}

VocabLayout vocab_layout(const vo_shape* s, const vo_teacher* t) {
  VocabLayout L;
  const int64_t N = s->N, H = s->H, V = s->V;
  L.f32 = s->dtype == AS_F32;
  L.g_bf16 = s->grad_dtype == AS_BF16;
  L.h_terms = L.f32 ? 3 : 1;
  L.dl_terms = L.g_bf16 ? 2 : 3;
  L.ldH = round_up(H, 8);
  L.strips = (int)((V + kVocabStrip - 1) / kVocabStrip);
  L.groups = (int)((N + kVocabGroup - 1) / kVocabGroup);
  const int64_t w_col = L.f32 ? L.ldH * 6 : 0;   // bytes of a column's terms of W
  // forward
  L.few = vocab_few_rows((int)N, (int)H, L.f32, t != nullptr);
  L.t_fwd = logits_tile(N, V, L.ldH, L.h_terms);
  const int64_t stat_col = (N * 16 + 63) / 64;
  L.fwd_cols = L.few ? round_up(V, kPieceColumns) : piece_columns(V, stat_col > w_col ? stat_col : w_col);
  // backward
  L.few_bwd = vocab_few_bwd_rows((int)N, (int)H, (int)V, L.f32, L.g_bf16);
  const int64_t dl_col = N * 2 * L.dl_terms;
  L.bwd_cols = piece_columns(V, dl_col > w_col ? dl_col : w_col);
  // bf16 gradients of many rows, pieces of twice the columns that are whole rounds of 256 x 256 tiles of dW: those kernels, one behind the
  // other; a split of dh's, a term at a time, is chosen by the device from the rows that there are.  us, the whole call, joint launch of
  // 128 x 128 tiles / this: 4096 x 1024 x 32000 1667 / 1533, 5120 2246 / 1995, 6400 with 30 % padding 2103 / 1846, 8192 x 1024 x 16000 with
  // 30 % 1187 / 1218, 16384 x 2048 x 128000 with 25 % 36070 / 34080; below the line 2257 x 1000 x 32003 with 30 % 759 / 950.
  if (L.dl_terms == 2 && N >= 4096) {
    const int64_t cols = piece_columns(V, N * 2), ldd = round_up(cols < V ? cols : V, 8), most = kPieceBytes / (N * L.ldH * 4);
    const int64_t tiles = ((ldd + 255) / 256) * ((H + 255) / 256), rounds = (tiles + 255) / 256;
    // two rounds of dh's tiles and more: not split, both terms in one launch (split / not, 16384 x 2048 x 128000 with 25 % padding 35010 / 34080
    // us, 16384 x 2048 x 32000 11500 / 10840)
    const bool split = ((N + 255) / 256) * ((L.ldH + 255) / 256) < 512;
    if (tiles * 8 >= rounds * 256 * 7 && (!split || most >= 2)) {
      L.apart = true;
      L.bwd_cols = cols;
      L.p_dw = {kTile256, 1};
      L.p_dh = {kTile256, !split ? 1 : most < 4 ? (int)most : 4};
    }
  }
  L.ldd = round_up(L.bwd_cols < V ? L.bwd_cols : V, 8);
  L.t_bwd = logits_tile(N, L.ldd, L.ldH, L.h_terms);
  // The two products of a piece in one launch of 128 x 128 tiles, the blocks of dh first, whose reductions are the longer ones: as
  // launches of their own, each is some part of a round of the compute units too long.  A reduction is split where one of its
  // blocks would otherwise take longer than half of all blocks' share of a compute unit's two places.
  const int n_dw = pair_count(L.dl_terms, L.h_terms);
  const int64_t k_dw = n_dw * ((N + 63) / 64), k_dh = n_dw * ((L.ldd + 63) / 64);
  if (!L.apart && N > 256) {
    const int64_t b_dw = ((L.ldd + 127) / 128) * ((H + 127) / 128), b_dh = ((N + 127) / 128) * ((L.ldH + 127) / 128);
    int64_t share = (b_dw * k_dw + b_dh * k_dh + 511) / 512;
    if (share < 8) share = 8;
    auto splits = [&](int64_t k) {
      const int64_t n = (2 * k + share - 1) / share;
      return whole_splits((int)k, n < 32 ? (int)n : 32);
    };
    L.p_dw = {kTile128, splits(k_dw)};
    L.p_dh = {kTile128, splits(k_dh)};
  } else if (!L.apart) {
    L.p_dw = gemm_plan((int)L.ldd, (int)H, (int)k_dw * 64, 1, true, true, true, true);
    L.p_dh = gemm_plan((int)N, (int)L.ldH, (int)k_dh * 64, 1, true, true, true, true);
    if (L.p_dw.tile == kTile256) L.p_dw = {kTile128, 1};
    if (L.p_dh.tile == kTile256) L.p_dh = {kTile128, 1};
  }
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += upv(bytes);
    return o;
  };
  const int64_t Np = round_up(N, kVocabRowPad);
  L.rows = take(N * 4);
  L.row_pos = take(N * 4);
  L.chunk_words = take(N > kRowsDirect ? (N + kRowsChunk - 1) / kRowsChunk * 4 : 0);
  L.y = take(Np * 4);
  L.n_act = take(16);
  L.ticket = take(16);
  L.hc = take((size_t)L.h_terms * N * L.ldH * 2);
  L.lse = take(Np * 4);
  L.at_word = take(N * 4);
  L.loss_ws = take(N * 4);
  L.run = take(L.fwd_cols < V ? N * 16 : 0);
  L.lse_tau = L.distill_ws = L.runs = L.ent = L.ent_p = L.ent_l = L.place = L.p_log_p = L.seen = 0;
  if (t) {
    const size_t entries = (size_t)L.groups * kVocabGroup * t->K;
    L.lse_tau = take(Np * 4);
    L.distill_ws = take(N * 4);
    L.runs = take((size_t)L.groups * (L.strips + 1) * 4);
    L.ent = take(entries * 4);
    L.ent_p = take(entries * 4);
    L.ent_l = take(entries * 4);
    L.place = take((size_t)N * t->K * 4);
    L.p_log_p = take(N * 4);
    L.seen = take(N * 4);
  }
  L.w_kept = L.f32 && !L.few && !L.few_bwd && V * w_col <= kPieceBytes;
  L.w_fwd = L.w_bwd = take(L.w_kept ? (size_t)V * w_col : 0);
  const size_t area = off;
  const int64_t parts = L.fwd_cols / kVocabStatCols;
  L.stat = take((size_t)parts * N * 8);
  L.stat_tau = take(t ? (size_t)parts * N * 4 : 0);
  L.stat_idx = take((size_t)parts * N * 4);
  if (!L.w_kept && !L.few) L.w_fwd = take((size_t)L.fwd_cols * w_col);
  size_t end = off;
  off = area;
  if (L.few_bwd) {
    L.dh_acc = take(vocab_few_bwd_bytes((int)N, (int)H, (int)V));
    L.total = off > end ? off : end;
    return L;
  }
  L.dl = take((size_t)L.dl_terms * N * L.ldd * 2);
  if (!L.w_kept) L.w_bwd = take((size_t)L.bwd_cols * w_col);
  L.ld_sums = round_up(V, 4);
  L.col_sums = take((size_t)((N + vocab_sum_rows(L.t_bwd) - 1) / vocab_sum_rows(L.t_bwd)) * L.ld_sums * 4);
  L.dh_acc = take((size_t)N * L.ldH * 4);
  L.partial_dw = take(gemm_partial_bytes((int)L.ldd, (int)H, 1, L.p_dw.splits));
  L.partial_dh = take(gemm_partial_bytes((int)N, (int)L.ldH, 1, L.p_dh.splits));
  L.total = off > end ? off : end;
  return L;
}

bool al16v(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

as_status check_shape(const vo_shape* s, const vo_teacher* t, bool wants_teacher) {
  if (!s) return set_error(AS_ERR_NULL, "shape is NULL");
  if (wants_teacher && !t) return set_error(AS_ERR_NULL, "teacher is NULL");
  if (!types_ok(s)) return set_error(AS_ERR_DTYPE, "vocabulary loss: dtype %d with grad_dtype %d", s->dtype, s->grad_dtype);
  if (!shape_ok(s))
    return set_error(AS_ERR_SHAPE, "bad shape N=%d H=%d V=%d pad_id=%d grad_scale=%g", s->N, s->H, s->V, s->pad_id, (double)s->grad_scale);
  if (t && !teacher_ok(s, t))
    return set_error(AS_ERR_SHAPE, "bad teacher K=%d temperature=%g scale=%g (V=%d)", t->K, (double)t->temperature, (double)t->scale, s->V);
  if (s->dtype == AS_BF16 && s->H % 8 != 0) return set_error(AS_ERR_ALIGN, "AS_BF16 requires H %% 8 == 0 (H=%d)", s->H);
  return AS_OK;
}
as_status check_workspace(const VocabLayout& L, const void* ws, size_t bytes) {
  if (bytes < L.total) return set_error(AS_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", bytes, L.total);
  if (!al16v(ws)) return set_error(AS_ERR_ALIGN, "workspace is not 16-byte aligned");
  return AS_OK;
}

struct Ws {
  unsigned char* base;
  template <typename T> T* at(size_t off) const { return reinterpret_cast<T*>(base + off); }
};

// h W_piece^T for the columns [v0, v0 + cols), with the terms of W in `planes` where there are any
GemmArgs logits_product(const vo_shape* s, const VocabLayout& L, const Ws& w, const void* W, const uint16_t* planes, int64_t plane,
                        int64_t v0, int cols) {
  GemmArgs g;
  int pairs[kMaxSeg][2];
  const int n = term_pairs(L.h_terms, L.h_terms, pairs);
  const uint16_t* hc = w.at<uint16_t>(L.hc);
  const int64_t h_plane = (int64_t)s->N * L.ldH;
  for (int i = 0; i < n; ++i) {
    const uint16_t* b = L.f32 ? planes + pairs[i][1] * plane : reinterpret_cast<const uint16_t*>(W) + v0 * s->H;
    g.seg(hc + pairs[i][0] * h_plane, L.ldH, 0, b, L.ldH, 0, (int)L.ldH);
  }
  g.M = s->N;
  g.N = cols;
  g.ldc = round_up(cols, 8);
  g.M_dev = w.at<int32_t>(L.n_act);
  return g;
}
const void* bias_at(const vo_shape* s, const void* b, int64_t v0) {
  if (!b) return nullptr;
  return reinterpret_cast<const unsigned char*>(b) + v0 * (s->dtype == AS_F32 ? 4 : 2);
}

// dl is kept relative to alpha, the larger of its factors g and s tau: its terms stay in bf16's range whatever these are.
struct DlUnit {
  float alpha, a1, a2;   // dl / alpha = a1 (..) + a2 (..)
};
DlUnit dl_unit(float g, float c2) {
  if (std::fabs(g) >= std::fabs(c2)) return {g, 1.f, g == 0.f ? 0.f : c2 / g};
  return {c2, g / c2, 1.f};
}

as_status hip_fail(hipError_t e, const char* what) { return set_error(AS_ERR_HIP, "%s: %s", what, hipGetErrorString(e)); }

as_status forward(const vo_shape* s, const vo_teacher* t, const void* h, const void* W, const void* b, const int32_t* targets,
                  const int32_t* teacher_ids, const float* teacher_logits, float* loss_sum, int32_t* n_tok, float* distill_sum,
                  float* tok_loss, float* tok_distill, int32_t* argmax, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!h || !W || !targets || !loss_sum || !n_tok || !workspace) return set_error(AS_ERR_NULL, "a required pointer is NULL");
  if (t && (!teacher_ids || !teacher_logits || !distill_sum)) return set_error(AS_ERR_NULL, "a required pointer is NULL");
  const VocabLayout L = vocab_layout(s, t);
  const as_status rc = check_workspace(L, workspace, workspace_bytes);
  if (rc != AS_OK) return rc;
  for (const void* p : {h, W, b, (const void*)targets, (const void*)teacher_ids, (const void*)teacher_logits, (const void*)loss_sum,
                        (const void*)n_tok, (const void*)distill_sum, (const void*)tok_loss, (const void*)tok_distill, (const void*)argmax})
    if (!al16v(p)) return set_error(AS_ERR_ALIGN, "a pointer is not 16-byte aligned");
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const Ws w{reinterpret_cast<unsigned char*>(workspace)};
  const int N = s->N;
  const int64_t h_plane = (int64_t)N * L.ldH;

  VocabRows r{};
  r.h = h;
  r.f32 = L.f32;
  r.targets = targets;
  r.N = N;
  r.H = s->H;
  r.V = s->V;
  r.pad_id = s->pad_id;
  r.row_pos = w.at<int32_t>(L.row_pos);
  r.rows = w.at<int32_t>(L.rows);
  r.y = w.at<int32_t>(L.y);
  r.n_act = w.at<int32_t>(L.n_act);
  r.hc = w.at<uint16_t>(L.hc);
  r.ldH = L.ldH;
  r.plane = h_plane;
  r.tok_loss = tok_loss;
  r.tok_distill = tok_distill;
  r.argmax = argmax;
  r.ticket = w.at<int32_t>(L.ticket);
  r.chunk_words = N > kRowsDirect ? w.at<int32_t>(L.chunk_words) : nullptr;
  hipError_t e = L.few && !t ? hipSuccess : launch_vocab_rows(r, st);
  if (e != hipSuccess) return hip_fail(e, "rows of words");

  const float inv_tau = t ? 1.f / t->temperature : 1.f;
  if (t) {
    VocabTeacher q{};
    q.ids = teacher_ids;
    q.logits = teacher_logits;
    q.N = N;
    q.K = t->K;
    q.V = s->V;
    q.inv_tau = inv_tau;
    q.rows = r.rows;
    q.n_act = r.n_act;
    q.runs = w.at<int32_t>(L.runs);
    q.ent = w.at<uint32_t>(L.ent);
    q.ent_p = w.at<float>(L.ent_p);
    q.place = w.at<int32_t>(L.place);
    q.p_log_p = w.at<float>(L.p_log_p);
    q.seen = w.at<int32_t>(L.seen);
    q.strips = L.strips;
    e = launch_vocab_teacher(q, st);
    if (e != hipSuccess) return hip_fail(e, "teacher's lists");
  }

  VocabFinish f{};
  f.stat = w.at<float2>(L.stat);
  f.stat_tau = t ? w.at<float>(L.stat_tau) : nullptr;
  f.stat_idx = argmax ? w.at<int32_t>(L.stat_idx) : nullptr;
  f.ldr = N;
  f.run = w.at<float4>(L.run);
  f.at_word = w.at<float>(L.at_word);
  f.rows = r.rows;
  f.n_act = r.n_act;
  f.N = N;
  f.lse = w.at<float>(L.lse);
  f.loss_ws = w.at<float>(L.loss_ws);
  f.tok_loss = tok_loss;
  f.tok_distill = tok_distill;
  f.argmax = argmax;
  f.loss_sum = loss_sum;
  f.distill_sum = distill_sum;
  f.n_tok = n_tok;
  f.ticket = r.ticket;
  f.inv_tau = inv_tau;
  if (t) {
    f.lse_tau = w.at<float>(L.lse_tau);
    f.distill_ws = w.at<float>(L.distill_ws);
    f.K = t->K;
    f.tau2 = t->temperature * t->temperature;
    f.place = w.at<int32_t>(L.place);
    f.seen = w.at<int32_t>(L.seen);
    f.ent_p = w.at<float>(L.ent_p);
    f.ent_l = w.at<float>(L.ent_l);
    f.p_log_p = w.at<float>(L.p_log_p);
  }
  for (int64_t v0 = 0; v0 < s->V; v0 += L.fwd_cols) {
    const int cols = (int)(s->V - v0 < L.fwd_cols ? s->V - v0 : L.fwd_cols);
    uint16_t* planes = w.at<uint16_t>(L.w_fwd) + (L.w_kept ? v0 * L.ldH : 0);
    const int64_t plane = (L.w_kept ? s->V : L.fwd_cols) * L.ldH;
    if (L.few) {
      // (W as it is)
    } else if (L.f32 && L.w_kept && v0 == 0) {
      e = launch_vocab_terms(reinterpret_cast<const float*>(W), s->V, s->H, planes, L.ldH, plane, st);
      if (e != hipSuccess) return hip_fail(e, "terms of W");
    } else if (L.f32 && !L.w_kept) {
      e = launch_vocab_terms(reinterpret_cast<const float*>(W) + v0 * s->H, cols, s->H, planes, L.ldH, plane, st);
      if (e != hipSuccess) return hip_fail(e, "terms of W");
    }
    VocabEpi v{};
    v.v0 = (int32_t)v0;
    v.y = r.y;
    v.bias = bias_at(s, b, v0);
    v.bias_f32 = L.f32;
    v.inv_tau = inv_tau;
    v.stat = w.at<float2>(L.stat);
    v.stat_tau = w.at<float>(L.stat_tau);
    v.stat_idx = w.at<int32_t>(L.stat_idx);
    v.ldr = N;
    v.at_word = w.at<float>(L.at_word);
    v.runs = w.at<int32_t>(L.runs);
    v.ent = w.at<uint32_t>(L.ent);
    v.ent_l = w.at<float>(L.ent_l);
    v.strips = L.strips;
    e = L.few ? launch_vocab_few(r, v, W, argmax != nullptr, t != nullptr, st)
              : launch_gemm_vocab(logits_product(s, L, w, W, planes, plane, v0, cols), L.t_fwd, v, 0, t != nullptr, argmax != nullptr, st);
    if (e != hipSuccess) return hip_fail(e, "statistics of the logits");
    const int part = L.few ? kVocabFewCols : kVocabStatCols;
    f.parts = (cols + part - 1) / part;
    f.first = v0 == 0;
    f.last = v0 + L.fwd_cols >= s->V;
    e = launch_vocab_finish(f, st);
    if (e != hipSuccess) return hip_fail(e, "losses");
  }
  return AS_OK;
}

as_status backward(const vo_shape* s, const vo_teacher* t, const void* W, const void* b, void* workspace, size_t workspace_bytes,
                   void* dh, void* dW, void* db, void* hip_stream) {
  if (!W || !workspace || !dh || !dW) return set_error(AS_ERR_NULL, "a required pointer is NULL");
  const VocabLayout L = vocab_layout(s, t);
  const as_status rc = check_workspace(L, workspace, workspace_bytes);
  if (rc != AS_OK) return rc;
  for (const void* p : {W, b, (const void*)dh, (const void*)dW, (const void*)db})
    if (!al16v(p)) return set_error(AS_ERR_ALIGN, "a pointer is not 16-byte aligned");
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const Ws w{reinterpret_cast<unsigned char*>(workspace)};
  const int N = s->N, H = s->H;
  const int32_t* n_act = w.at<int32_t>(L.n_act);
  const int64_t h_plane = (int64_t)N * L.ldH, dl_plane = (int64_t)N * L.ldd;
  const int64_t w_plane = (L.w_kept ? s->V : L.bwd_cols) * L.ldH;
  uint16_t* dl = w.at<uint16_t>(L.dl);
  const size_t ge = L.g_bf16 ? 2 : 4;
  int pairs[kMaxSeg][2];
  const int n = term_pairs(L.dl_terms, L.h_terms, pairs);
  const float c2 = t ? t->scale * t->temperature : 0.f;
  const DlUnit unit = dl_unit(s->grad_scale, c2);
  const float alpha = unit.alpha;
  hipError_t e;
  if (L.few_bwd) {
    VocabFewBwd f{};
    f.f32 = L.f32;
    f.g_bf16 = L.g_bf16;
    f.teacher = t != nullptr;
    f.hc = w.at<uint16_t>(L.hc);
    f.ldH = L.ldH;
    f.plane = h_plane;
    f.n_act = n_act;
    f.row_pos = w.at<int32_t>(L.row_pos);
    f.N = N;
    f.H = H;
    f.V = s->V;
    f.W = W;
    f.epi.y = w.at<int32_t>(L.y);
    f.epi.bias = b;
    f.epi.lse = w.at<float>(L.lse);
    f.epi.lse_tau = w.at<float>(L.lse_tau);
    f.epi.a1 = s->grad_scale;
    f.epi.a2 = c2;
    f.epi.inv_tau = t ? 1.f / t->temperature : 1.f;
    f.epi.runs = w.at<int32_t>(L.runs);
    f.epi.ent = w.at<uint32_t>(L.ent);
    f.epi.ent_p = w.at<float>(L.ent_p);
    f.epi.strips = L.strips;
    f.dh = dh;
    f.dW = dW;
    f.db = db;
    f.dh_part = w.at<float>(L.dh_acc);
    e = launch_vocab_few_bwd(f, st);
    return e == hipSuccess ? AS_OK : hip_fail(e, "gradients of a few rows");
  }
  for (int64_t v0 = 0; v0 < s->V; v0 += L.bwd_cols) {
    const int cols = (int)(s->V - v0 < L.bwd_cols ? s->V - v0 : L.bwd_cols);
    uint16_t* planes = w.at<uint16_t>(L.w_bwd) + (L.w_kept ? v0 * L.ldH : 0);
    if (L.f32 && !L.w_kept) {
      e = launch_vocab_terms(reinterpret_cast<const float*>(W) + v0 * H, cols, H, planes, L.ldH, w_plane, st);
      if (e != hipSuccess) return hip_fail(e, "terms of W");
    }
    VocabEpi v{};
    v.v0 = (int32_t)v0;
    v.y = w.at<int32_t>(L.y);
    v.bias = bias_at(s, b, v0);
    v.bias_f32 = L.f32;
    v.inv_tau = t ? 1.f / t->temperature : 1.f;
    v.runs = w.at<int32_t>(L.runs);
    v.ent = w.at<uint32_t>(L.ent);
    v.ent_p = w.at<float>(L.ent_p);
    v.strips = L.strips;
    v.lse = w.at<float>(L.lse);
    v.lse_tau = w.at<float>(L.lse_tau);
    v.a1 = unit.a1;
    v.a2 = unit.a2;
    v.dl = dl;
    v.ldd = L.ldd;
    v.plane = dl_plane;
    v.col_sums = db ? w.at<float>(L.col_sums) + v0 : nullptr;
    v.ld_sums = L.ld_sums;
    e = launch_gemm_vocab(logits_product(s, L, w, W, planes, w_plane, v0, cols), L.t_bwd, v, L.dl_terms, t != nullptr, false, st);
    if (e != hipSuccess) return hip_fail(e, "derivative of the logits");
    GemmArgs g[2];   // dW_piece = dl^T h, dh += dl W_piece
    for (int i = 0; i < n; ++i) {
      const uint16_t* a = dl + pairs[i][0] * dl_plane;
      const uint16_t* wb = L.f32 ? planes + pairs[i][1] * w_plane : reinterpret_cast<const uint16_t*>(W) + v0 * H;
      g[0].seg(a, L.ldd, 0, w.at<uint16_t>(L.hc) + pairs[i][1] * h_plane, L.ldH, 0, N);
      g[1].seg(a, L.ldd, 0, wb, L.ldH, 0, cols);
    }
    g[0].a_kc = g[0].b_kc = g[1].b_kc = false;
    g[0].M = cols;
    g[0].N = H;
    g[0].C = reinterpret_cast<unsigned char*>(dW) + (size_t)v0 * H * ge;
    g[0].ldc = H;
    g[0].c_bf16 = L.g_bf16;
    g[0].K_dev = n_act;
    g[0].alpha = alpha;
    g[0].splits = L.p_dw.splits;
    g[0].partial = w.at<float>(L.partial_dw);
    g[1].M = N;
    g[1].N = (int)L.ldH;
    g[1].C = w.at<float>(L.dh_acc);
    g[1].ldc = L.ldH;
    g[1].accumulate = v0 > 0;
    g[1].M_dev = n_act;
    g[1].splits = whole_splits(n * ((cols + 63) / 64), L.p_dh.splits);
    g[1].partial = w.at<float>(L.partial_dh);
    if (L.apart) {
      e = launch_gemm(g[0], true, L.p_dw.tile, st);
      if (L.p_dh.splits == 1 && e == hipSuccess) e = launch_gemm(g[1], true, L.p_dh.tile, st);
      for (int i = 0; i < n && L.p_dh.splits > 1 && e == hipSuccess; ++i) {
        GemmArgs one = g[1];
        one.A[0] = g[1].A[i];   // (h and W have one term, so every segment's B is the same)
        one.K[1] = 0;
        one.nseg = 1;
        one.accumulate = v0 > 0 || i > 0;
        one.splits = L.p_dh.splits;
        one.dyn_split = true;
        e = launch_gemm(one, true, L.p_dh.tile, st);
      }
      if (e != hipSuccess) return hip_fail(e, "dW and dh");
      continue;
    }
    const GemmTile tiles[2] = {L.p_dw.tile, L.p_dh.tile};
    const DbReduce no_sums = {nullptr, 0, 0, nullptr, nullptr, 1};   // (db is added up with the last pass)
    e = launch_gemm_joint(g, tiles, 2, true, st, &no_sums);
    if (e == hipErrorNotSupported) e = hipSuccess;
    else if (e == hipSuccess) continue;
    for (int i = 0; i < 2 && e == hipSuccess; ++i) e = launch_gemm(g[i], true, tiles[i], st);
    if (e != hipSuccess) return hip_fail(e, "dW and dh");
  }
  VocabOutGrads o{};
  o.src = w.at<float>(L.dh_acc);
  o.row_pos = w.at<int32_t>(L.row_pos);
  o.N = N;
  o.H = H;
  o.ld = L.ldH;
  o.dh = dh;
  o.sums = w.at<float>(L.col_sums);
  o.ld_sums = L.ld_sums;
  o.sum_rows = vocab_sum_rows(L.t_bwd);
  o.n_act = n_act;
  o.V = s->V;
  o.db = db;
  o.alpha = alpha;
  e = launch_vocab_out_grads(o, L.g_bf16, st);
  if (e != hipSuccess) return hip_fail(e, "dh and db");
  return AS_OK;
}

}  // namespace
}  // namespace asx

using namespace asx;

extern "C" size_t vocab_xent_workspace_bytes(const vo_shape* shape, const vo_teacher* teacher) {
  if (!shape || !types_ok(shape) || !shape_ok(shape) || (shape->dtype == AS_BF16 && shape->H % 8 != 0)) return 0;
  if (teacher && !teacher_ok(shape, teacher)) return 0;
  return vocab_layout(shape, teacher).total;
}

extern "C" as_status vocab_xent_fwd(const vo_shape* shape, const void* h, const void* W, const void* b, const int32_t* targets,
                                    float* loss_sum, int32_t* n_tok, float* tok_loss, int32_t* argmax,
                                    void* workspace, size_t workspace_bytes, void* hip_stream) {
  const as_status rc = check_shape(shape, nullptr, false);
  if (rc != AS_OK) return rc;
  return forward(shape, nullptr, h, W, b, targets, nullptr, nullptr, loss_sum, n_tok, nullptr, tok_loss, nullptr, argmax, workspace,
                 workspace_bytes, hip_stream);
}
extern "C" as_status vocab_xent_bwd(const vo_shape* shape, const void* W, const void* b, void* workspace, size_t workspace_bytes,
                                    void* dh, void* dW, void* db, void* hip_stream) {
  const as_status rc = check_shape(shape, nullptr, false);
  if (rc != AS_OK) return rc;
  return backward(shape, nullptr, W, b, workspace, workspace_bytes, dh, dW, db, hip_stream);
}
extern "C" as_status vocab_distill_fwd(const vo_shape* shape, const vo_teacher* teacher, const void* h, const void* W, const void* b,
                                       const int32_t* targets, const int32_t* teacher_ids, const float* teacher_logits,
                                       float* loss_sum, int32_t* n_tok, float* distill_sum, float* tok_loss, float* tok_distill,
                                       void* workspace, size_t workspace_bytes, void* hip_stream) {
  const as_status rc = check_shape(shape, teacher, true);
  if (rc != AS_OK) return rc;
  return forward(shape, teacher, h, W, b, targets, teacher_ids, teacher_logits, loss_sum, n_tok, distill_sum, tok_loss, tok_distill,
                 nullptr, workspace, workspace_bytes, hip_stream);
}
extern "C" as_status vocab_distill_bwd(const vo_shape* shape, const vo_teacher* teacher, const void* W, const void* b,
                                       void* workspace, size_t workspace_bytes, void* dh, void* dW, void* db, void* hip_stream) {
  const as_status rc = check_shape(shape, teacher, true);
  if (rc != AS_OK) return rc;
  return backward(shape, teacher, W, b, workspace, workspace_bytes, dh, dW, db, hip_stream);
}
