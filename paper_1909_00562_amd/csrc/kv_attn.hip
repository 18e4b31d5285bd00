// Attention of each sequence's newest tokens over its paged cache (entry point and kernels).
//
// The queries that share a head of the cache are the rows of a product of 16 columns: S^T = K Q^T and O^T = V^T P^T, one pass over
// keys and values with the running maximum and sum of the softmax.  Bound by memory: each cached value is read once; at four
// queries to a head the products are 16 operations for each of a key's and a value's bf16 elements.
//
// Nothing goes through LDS but what waves of a block join at the end.  A wave takes tiles of 16 tokens.  K's fragments are read as they
// lie.  S^T leaves lane (c, g) = (lane & 15, lane >> 4) with the scores of row c and of tokens 4g .. 4g + 3, which is how the next
// product takes P^T, with its reduction index numbered to suit: the same lane's V fragment holds the same tokens.  Of V a lane reads
// consecutive columns of these tokens, and fragments are made of them in its own registers: columns of O^T are numbered to suit.
// Row c's factor of O^T is then the lane's own too.
//
// Work is cut by what the sequences hold: all (sequence, head, chunk of tokens) are numbered in one row, and a block takes a run of
// equal length.  What is left of a (sequence, head) that several blocks share goes to the workspace, joined by a second launch.
#include "kv_cache.h"

#include <cmath>
#include <type_traits>

#include "common.h"
#include "lds_limit.h"
#include "status.h"

namespace asx {
namespace {

typedef uint32_t au32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t au32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// The table is read past the vector memory's counter: a page looked up among the loads of a step would have to wait for those ahead of it.
typedef __attribute__((address_space(4))) int32_t scalar_int32_t;
constexpr int kLongRun = 8;            // chunks
constexpr int kLeastChunk = 16;
constexpr int kWholeSteps = 4;
constexpr uint32_t kAttnOob = 0x80000000u;
constexpr float kLog2e = 1.4426950408889634f;

struct KvAttnDev {
  const void *q, *k_pages, *v_pages;
  const float *k_scales, *v_scales;
  const int32_t *table, *lengths;
  void* out;
  float* lse;
  float *part, *part_ml;   // [slot][row][D], [slot][row][2]: sums relative to the maximum; the largest score ahead of its scale, and the sum of weights
  int64_t ld_q;
  int32_t B, T, heads, G, D, R;        // R = T G rows of a head
  int32_t tile_waves, tok_waves, row_groups, group_rows;   // tiles of 16 rows of a block (1 to 4); waves of each, sharing tokens; groups of a block's tiles; rows of a group
  KvMagic by_tile_waves, by_quads;     // divisions by tile_waves and by D / 4
  int32_t page, page_tiles, pages, max_pages, max_len, window;
  KvMagic magic;                       // of page_tiles
  int32_t chunk;                       // tokens of a chunk
  int32_t split;                       // 0: a block per (sequence, head, row group), no second launch
  float scale, scale_log2;             // magnitudes, the second one times log2(e): a negative scale's sign goes into the queries
  int32_t no_q;                        // queries count as 0
  uint32_t q_sign;                     // exclusive-ored onto pairs of bf16 or onto floats
};

// ---- which tokens -----------------------------------------------------------------
struct SeqSpan {
  int32_t len, base, chunks;   // tokens; the first one that is looked at, rounded down to a tile; chunks from there
};
__device__ __forceinline__ SeqSpan seq_span(const KvAttnDev& a, int b) {
  SeqSpan s;
  int32_t n = a.lengths[b];
  n = n < 0 ? 0 : n > a.max_len ? a.max_len : n;
  const int32_t first = a.window > 0 ? n - a.T + 1 - a.window : 0;
  s.len = n;
  s.base = first > 0 ? first & ~(kKvTile - 1) : 0;
  s.chunks = (n - s.base + a.chunk - 1) / a.chunk;
  return s;
}

// How the chunks of all (sequence, head, row group) are given to the blocks.
struct Cut {
  int32_t total;   // chunks
  int32_t per;     // of a block, at most
  bool pieces;     // a block has one piece of one (sequence, head, row group), those of one sequence being of the same length; else a run
                   // of `per` chunks, whatever they are of
  // a sequence's pieces, or chunks, for each of its heads and row groups
  __device__ __forceinline__ int32_t units(int32_t chunks) const { return pieces ? (chunks + per - 1) / per : chunks; }
};
// A run that ends one sequence's head and begins the next one's reads two sets of queries and writes two results, which costs as much as
// some chunks do: short runs are pieces instead, if pieces that are not full leave no more blocks without work than that.
// us, kernels: 24 sequences of two heads, 1004 tokens seen by 40 rows, e4m3, runs / pieces 23.3 / 17.8.
__device__ __forceinline__ Cut cut_of(const KvAttnDev& a, int32_t chunks, int blocks) {
  const int32_t hr = a.heads * a.row_groups;
  Cut c;
  c.total = chunks * hr;
  c.per = (c.total + blocks - 1) / blocks;
  if (c.per < 1) c.per = 1;
  c.pieces = false;
  const int64_t pairs = (int64_t)a.B * hr;
  if (2 * pairs <= blocks) {
    const int32_t left = blocks - (int32_t)pairs, per = (c.total + left - 1) / left;   // sum of (n + per - 1) / per <= total / per + pairs
    if (per < kLongRun) {
      c.per = per < 1 ? 1 : per;
      c.pieces = true;
    }
  }
  return c;
}
template <int WAVES> __device__ __forceinline__ int32_t sum_of_waves(int32_t n, int32_t* s_sum) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) n += s_sum[w];
  return n;
}
template <int WAVES> __device__ __forceinline__ Cut cut_all(const KvAttnDev& a, int blocks, int32_t* s_sum) {
  int32_t n = 0;
  for (int b = threadIdx.x; b < a.B; b += WAVES * 64) n += seq_span(a, b).chunks;
  return cut_of(a, sum_of_waves<WAVES>(n, s_sum), blocks);
}
// A block's work: `left` chunks from `chunk` on of sequence b's head and row group hr; 0: none.
struct Run {
  int32_t b, hr, chunk, left;
  int32_t per;   // Cut's
};
// lanes' sums up to and including their own
__device__ __forceinline__ int32_t scan_lanes(int32_t n) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t x = __shfl_up(n, o, 64);
    if (lane >= o) n += x;
  }
  return n;
}
// Up to 64 sequences a wave cuts by itself, a lane for each: its chunks, and its units for all heads with those of the sequences ahead.
struct LaneCut {
  Cut cut;
  int32_t chunks, own, ahead;
};
__device__ __forceinline__ LaneCut cut_lanes(const KvAttnDev& a, int blocks) {
  const int lane = threadIdx.x & 63;
  LaneCut r;
  r.chunks = lane < a.B ? seq_span(a, lane).chunks : 0;
  const int32_t hrs = a.heads * a.row_groups, upto = scan_lanes(r.chunks);
  r.cut = cut_of(a, __builtin_amdgcn_readlane(upto, 63), blocks);
  const int32_t units = r.cut.units(r.chunks);
  r.own = units * hrs;
  r.ahead = (r.cut.pieces ? scan_lanes(units) : upto) * hrs - r.own;
  return r;
}
// what a block does of sequence b, from unit `rest` of it on
__device__ __forceinline__ Run run_of(const Cut& c, int32_t b, int32_t n, int32_t rest, int32_t at) {
  Run r;
  r.b = b;
  r.per = c.per;
  const int32_t units = c.units(n);
  r.hr = rest / units;
  const int32_t unit = rest - r.hr * units;
  if (c.pieces) {
    const int32_t each = n / units, more = n - each * units;   // the first `more` pieces have one chunk more
    r.chunk = unit * each + (unit < more ? unit : more);
    r.left = each + (unit < more);
  } else {
    r.chunk = unit;
    r.left = c.total - at < c.per ? c.total - at : c.per;
  }
  return r;
}
template <int WAVES> __device__ __forceinline__ Run cut_run(const KvAttnDev& a, int32_t* s_sum, int32_t* s_found) {
  if (a.B <= 64) {
    const LaneCut l = cut_lanes(a, gridDim.x);
    const int32_t at = l.cut.pieces ? (int32_t)blockIdx.x : (int32_t)blockIdx.x * l.cut.per;
    const uint64_t here = __ballot(at >= l.ahead && at < l.ahead + l.own);
    if (!here) return {0, 0, 0, 0, 0};
    const int b = __builtin_ctzll(here);
    return run_of(l.cut, b, __builtin_amdgcn_readlane(l.chunks, b), at - __builtin_amdgcn_readlane(l.ahead, b), at);
  }
  const Cut c = cut_all<WAVES>(a, gridDim.x, s_sum);
  const int32_t hrs = a.heads * a.row_groups, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t at = c.pieces ? (int32_t)blockIdx.x : (int32_t)blockIdx.x * c.per;   // in units, as is what follows
  Run r = {0, 0, 0, 0, 0};
  int32_t carry = 0;
  bool found = false;
  for (int b0 = 0; b0 < a.B && !found; b0 += WAVES * 64) {
    const int b = b0 + threadIdx.x;
    const int32_t own = b < a.B ? c.units(seq_span(a, b).chunks) * hrs : 0;
    int32_t run = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int32_t x = __shfl_up(run, o, 64);
      if (lane >= o) run += x;
    }
    __syncthreads();
    if (lane == 63) s_sum[wave] = run;
    __syncthreads();
    int32_t ahead = carry + run - own;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int32_t x = s_sum[w];
      ahead += w < wave ? x : 0;
      carry += x;
    }
    if (at >= ahead && at < ahead + own) {
      s_found[0] = b;
      s_found[1] = ahead;
    }
    found = at < carry;
  }
  if (!found) return r;                   // (the same in all threads)
  __syncthreads();
  return run_of(c, s_found[0], seq_span(a, s_found[0]).chunks, at - s_found[1], at);
}

// ---- fragments --------------------------------------------------------------------
__device__ __forceinline__ bf16x8_t as_frag(au32x4_t x) { return __builtin_bit_cast(bf16x8_t, x); }
__device__ __forceinline__ uint32_t top_halves(float lo, float hi) {   // two floats that bf16 holds
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
}

// bytes 2 HIGH and 2 HIGH + 1 of a word of e4m3 codes as bf16, which holds them
template <bool HIGH> __device__ __forceinline__ uint32_t e4m3_to_bf16(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HIGH));
}
__device__ __forceinline__ void int8_to_floats(uint32_t w, float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
}

// offsets from `bytes` on read as 0
__device__ __forceinline__ __amdgpu_buffer_rsrc_t attn_rsrc(const void* base, int32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}
// the larger of a lane's and of those 16, 32 and 48 lanes away
__device__ __forceinline__ float max_of_rows(float x) {
  const uint32_t a = __builtin_bit_cast(uint32_t, x);
  const auto p = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t p0 = p[0], p1 = p[1];
  const uint32_t c = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, p0), __builtin_bit_cast(float, p1)));
  const auto q = __builtin_amdgcn_permlane32_swap(c, c, false, false);
  const uint32_t q0 = q[0], q1 = q[1];
  return fmaxf(__builtin_bit_cast(float, q0), __builtin_bit_cast(float, q1));
}

// What a cache type's tiles look like.  TYPE: kc_type, F32Q: queries and results are float, DP: the head's width up to which it serves.
template <int TYPE, bool F32Q, int DP> struct Form {
  static constexpr bool kF32 = TYPE == KC_F32, kCoded = TYPE == KC_INT8 || TYPE == KC_E4M3;
  static constexpr int kBytes = kF32 ? 4 : kCoded ? 1 : 2;
  static constexpr int kTiles = kF32 ? 1 : 2;                       // of a step
  // Waves on a SIMD that registers allow: a wave holds a step's K and V, the queries and O^T in them.
  static constexpr int kOnSimd = DP > 128 ? 1 : DP > 64 || (TYPE != KC_F32 && (TYPE != KC_INT8 || F32Q)) ? 2 : 4;
  static constexpr int kQTerms = kF32 || !F32Q ? 1 : 3, kPTerms = kF32 ? 1 : F32Q ? 3 : 2;
  static constexpr int kKLoads = DP * kBytes / 64;                  // 16-byte loads of a lane for a tile of K
  static constexpr int kKElems = 16 / kBytes;                       // elements of each: D index (load * 4 + g) * kKElems + i
  // V: columns (half * 16 + c) * kVW + i of a token
  static constexpr int kVAll = DP / 16;                             // columns of a lane
  static constexpr int kVW = kCoded ? kVAll : kF32 ? 4 : (kVAll < 8 ? kVAll : 8);
  static constexpr int kVHalves = kVAll / kVW;
  static constexpr int kVDwords = kVW * kBytes / 4;
  // Values may be infinities or NaN: bits of theirs in a word, which no other value sets (an exponent of ones and one more), all bits of
  // theirs, and a word of ones.
  static constexpr bool kCanBeOdd = TYPE != KC_INT8;
  static constexpr uint32_t kOnes = kF32 ? 0x3f800000u : kCoded ? 0x38383838u : 0x3f803f80u;
  static __device__ __forceinline__ uint32_t odd(uint32_t w) {
    if constexpr (kF32) return ((w & 0x7f800000u) + 0x00800000u) & 0x80000000u;
    else if constexpr (kCoded) return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    else return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  }
  static __device__ __forceinline__ uint32_t odd_bits(uint32_t w) {
    const uint32_t x = odd(w) >> (kF32 ? 31 : kCoded ? 7 : 15);
    if constexpr (kF32) return 0u - x;
    else return (x << (kCoded ? 8 : 16)) - x;
  }
};

template <int N> __device__ __forceinline__ void buffer_load(__amdgpu_buffer_rsrc_t rs, uint32_t off, uint32_t (&x)[N]) {
  static_assert(N == 1 || N == 2 || N == 4);
  if constexpr (N == 4) {
    const au32x4_t q = __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = q[i];
  } else if constexpr (N == 2) {
    const au32x2_t q = __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0);
    x[0] = q[0];
    x[1] = q[1];
  } else {
    x[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0);
  }
}

// ---- the kernel -------------------------------------------------------------------
template <int TYPE, bool F32Q, int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64, (Form<TYPE, F32Q, DP>::kOnSimd)) void kv_attn_kernel(KvAttnDev a) {
  using F = Form<TYPE, F32Q, DP>;
  constexpr int NT = F::kTiles, NO = DP / 16, STEP = NT * kKvTile, LD = DP + 4;
  extern __shared__ float lds[];          // [waves][16 rows][LD], and their maxima and sums
  float* lds_ml = lds + WAVES * 16 * LD;
  __shared__ int32_t s_sum[WAVES], s_found[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int tok_wave = kv_div(wave, a.by_tile_waves), row_wave = wave - tok_wave * a.tile_waves, tok_waves = a.tok_waves;   // (some waves may be left over)

  // a lane's part of a tile of K and of V; behind a row's end: out of every range
  uint32_t k_off[F::kKLoads], v_off[4][F::kVHalves];
  const int32_t row_bytes = a.D * F::kBytes;
  const uint32_t k_at = c * row_bytes + g * 16, v_at = g * 4 * row_bytes + c * F::kVW * F::kBytes;
#pragma unroll
  for (int j = 0; j < F::kKLoads; ++j) k_off[j] = (j * 4 + g) * F::kKElems < a.D ? k_at + j * 64 : kAttnOob;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int h = 0; h < F::kVHalves; ++h)
      v_off[i][h] = (h * 16 + c) * F::kVW < a.D ? v_at + i * row_bytes + h * 16 * F::kVW * F::kBytes : kAttnOob;

  // this block's run of chunks
  int32_t b, hr, chunk, left;             // sequence, (head, row group), first chunk there, chunks left
  if (a.split) {
    const Run run = cut_run<WAVES>(a, s_sum, s_found);
    if (run.left <= 0) return;
    b = run.b;
    hr = run.hr;
    chunk = run.chunk;
    left = run.left;
  } else {
    b = blockIdx.x;
    hr = blockIdx.y;
    chunk = 0;
    left = 0;                             // (all there are)
  }
  b = __builtin_amdgcn_readfirstlane(b);
  hr = __builtin_amdgcn_readfirstlane(hr);
  chunk = __builtin_amdgcn_readfirstlane(chunk);
  left = __builtin_amdgcn_readfirstlane(left);

  do {
    const SeqSpan span = seq_span(a, b);
    const int32_t len = span.len;
    const int head = a.row_groups == 1 ? hr : hr / a.row_groups, group = hr - head * a.row_groups;
    const int32_t here = a.split ? (left < span.chunks - chunk ? left : span.chunks - chunk) : span.chunks;
    const int32_t tok0 = span.base + chunk * a.chunk;
    int32_t tok1 = tok0 + here * a.chunk;
    if (tok1 > len) tok1 = len;
    const bool whole = here == span.chunks;

    // the row of this lane's column of S^T and O^T
    const int row0 = (group * a.tile_waves + row_wave) * 16, row = row0 + c;
    const bool row_there = row < a.R;
    const int t = a.T == 1 || !row_there ? 0 : row / a.G, gq = row - t * a.G;
    const int32_t hi = row_there ? len - a.T + t : -1, lo = a.window > 0 ? hi - a.window + 1 : 0;
    // tokens that all rows of all t see
    const int32_t all_hi = len - a.T, all_lo = a.window > 0 ? len - a.window : 0;

    // the first tiles' pages are looked up ahead of everything else
    const scalar_int32_t* table = (const scalar_int32_t*)(uintptr_t)(a.table + (int64_t)b * a.max_pages);
    // the table's entry for the tile at pos (past the end: the last one)
    auto page_of = [&](int32_t pos) {
      const uint32_t tile = (uint32_t)(pos < len ? pos : len - 1) >> 4, col = kv_div(tile, a.magic);
      return table[col];
    };
    const int32_t stride = tok_waves * STEP;
    int32_t pos = tok0 + tok_wave * STEP;
    int32_t id[NT], id_next[NT];
    const bool any_steps = tok_wave < tok_waves && pos < tok1 && row0 < a.R;
    if (any_steps) {
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        id[u] = page_of(pos + u * kKvTile);
        id_next[u] = page_of(pos + stride + u * kKvTile);
      }
    }

    // queries
    constexpr int QF = F::kF32 ? DP / 16 : DP / 32;   // fragments: of 4 floats, or of 8 bf16
    float qf[F::kF32 ? QF : 1][4];
    bf16x8_t qb[F::kQTerms][F::kF32 ? 1 : QF];
    const bool q_there = row_there && !a.no_q;
    const int64_t q_at = ((int64_t)b * a.T + t) * a.ld_q + (int64_t)(head * a.G + gq) * a.D;
    if constexpr (F::kF32) {
#pragma unroll
      for (int j = 0; j < QF; ++j) {
        const int d = (j * 4 + g) * 4;
        f32x4_t v = {};
        if (q_there && d < a.D) v = *reinterpret_cast<const f32x4_t*>(reinterpret_cast<const float*>(a.q) + q_at + d);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = v[i];
          qf[j][i] = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) ^ a.q_sign);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < QF; ++j) {
        // codes: 16 of a load are two fragments
        const int d = F::kCoded ? (j / 2 * 4 + g) * 16 + j % 2 * 8 : (j * 4 + g) * 8;
        const bool there = q_there && d < a.D;
        if constexpr (!F32Q) {
          au32x4_t v = {};
          if (there) v = *reinterpret_cast<const au32x4_t*>(reinterpret_cast<const uint16_t*>(a.q) + q_at + d);
          qb[0][j] = as_frag(v ^ a.q_sign);
        } else {
          float v[8] = {};
          if (there) {
            const float* p = reinterpret_cast<const float*>(a.q) + q_at + d;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p[i];
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float rest = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v[i]) ^ a.q_sign);
#pragma unroll
            for (int s = 0; s < F::kQTerms; ++s) {
              const bf16_t x = (bf16_t)rest;
              qb[s][j][i] = x;
              rest -= (float)x;
            }
          }
        }
      }
    }

    f32x4_t o[NO] = {};
    float m = -INFINITY, l = 0.f;

    uint32_t kr[NT][F::kKLoads][4], vr[NT][4][F::kVHalves][F::kVDwords];
    float ks[NT][4], vs[NT][4];
    int32_t k_valid[NT];                  // tokens that there are of a tile: up to 16, 0 where there is no page
    // the tile's first row in the pool, and how many of its tokens there are
    auto place = [&](int32_t pos, int32_t id, int32_t& valid) {
      const uint32_t tile = (uint32_t)pos >> 4, col = kv_div(tile, a.magic);
      const bool there = (uint32_t)id < (uint32_t)a.pages;
      const int32_t n = there ? tok1 - pos : 0;
      valid = __builtin_amdgcn_readfirstlane(n < 0 ? 0 : n < kKvTile ? n : kKvTile);   // (a median of three is the vector unit's)
      return (int64_t)((there ? id : 0) * a.heads + head) * a.page + (int32_t)(tile - col * a.page_tiles) * kKvTile;
    };
    int64_t at_row[NT];                   // of the tiles whose keys were asked for last
    auto load_k = [&](int32_t pos, const int32_t (&id)[NT]) {
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        at_row[u] = place(pos + u * kKvTile, id[u], k_valid[u]);
        const auto rs = attn_rsrc(reinterpret_cast<const uint8_t*>(a.k_pages) + at_row[u] * row_bytes, k_valid[u] * row_bytes);
#pragma unroll
        for (int j = 0; j < F::kKLoads; ++j) buffer_load(rs, k_off[j], kr[u][j]);
        if constexpr (F::kCoded) {
          uint32_t x[4];
          buffer_load(attn_rsrc(a.k_scales + at_row[u], (k_valid[u] + 3) / 4 * 16), g * 16u, x);
#pragma unroll
          for (int i = 0; i < 4; ++i) ks[u][i] = __builtin_bit_cast(float, x[i]);
        }
      }
    };
    auto load_v = [&]() {                 // of the same tiles
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        const auto rs = attn_rsrc(reinterpret_cast<const uint8_t*>(a.v_pages) + at_row[u] * row_bytes, k_valid[u] * row_bytes);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int h = 0; h < F::kVHalves; ++h) buffer_load(rs, v_off[i][h], vr[u][i][h]);
        if constexpr (F::kCoded) {
          uint32_t x[4];
          buffer_load(attn_rsrc(a.v_scales + at_row[u], (k_valid[u] + 3) / 4 * 16), g * 16u, x);
#pragma unroll
          for (int i = 0; i < 4; ++i) vs[u][i] = __builtin_bit_cast(float, x[i]);
        }
      }
    };

    // The fragments of V^T, 16 columns after the other: use(j, fragment), or, of floats, use(j, i, value) for tokens i; raw(u, i, h, w) are
    // the loaded words, or others like them.
    auto columns = [&](auto raw, auto use) {
      if constexpr (F::kF32) {
#pragma unroll
        for (int j = 0; j < NO; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) use(j, i, __builtin_bit_cast(float, raw(0, i, j / F::kVW, j % F::kVW)));
      } else if constexpr (TYPE == KC_INT8) {
#pragma unroll
        for (int w = 0; w < F::kVDwords; ++w) {
          float x[2][4][4];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) int8_to_floats(raw(u, i, 0, w), x[u][i]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            use(w * 4 + e, as_frag(au32x4_t{top_halves(x[0][0][e], x[0][1][e]), top_halves(x[0][2][e], x[0][3][e]),
                                            top_halves(x[1][0][e], x[1][1][e]), top_halves(x[1][2][e], x[1][3][e])}));
        }
      } else if constexpr (TYPE == KC_E4M3) {
#pragma unroll
        for (int w = 0; w < F::kVDwords; ++w)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            // codes e and e + 1 of two tokens, side by side
            const uint32_t sel = e ? 0x07030602u : 0x05010400u;
            auto two = [&](int u, int i) { return __builtin_amdgcn_perm(raw(u, i + 1, 0, w), raw(u, i, 0, w), sel); };
            const uint32_t x[4] = {two(0, 0), two(0, 2), two(1, 0), two(1, 2)};
            use(w * 4 + e, as_frag(au32x4_t{e4m3_to_bf16<false>(x[0]), e4m3_to_bf16<false>(x[1]), e4m3_to_bf16<false>(x[2]), e4m3_to_bf16<false>(x[3])}));
            use(w * 4 + e + 1, as_frag(au32x4_t{e4m3_to_bf16<true>(x[0]), e4m3_to_bf16<true>(x[1]), e4m3_to_bf16<true>(x[2]), e4m3_to_bf16<true>(x[3])}));
          }
      } else {
#pragma unroll
        for (int h = 0; h < F::kVHalves; ++h)
#pragma unroll
          for (int e = 0; e < F::kVW; ++e) {
            const uint32_t sel = e % 2 ? 0x07060302u : 0x05040100u;
            auto two = [&](int u, int i) { return __builtin_amdgcn_perm(raw(u, i + 1, h, e / 2), raw(u, i, h, e / 2), sel); };
            use(h * F::kVW + e, as_frag(au32x4_t{two(0, 0), two(0, 2), two(1, 0), two(1, 2)}));
          }
      }
    };

    if (any_steps) {
      load_k(pos, id);
      load_v();
      for (; pos < tok1; pos += stride) {
        // S^T
        f32x4_t s[NT] = {};
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          if constexpr (F::kF32) {
#pragma unroll
            for (int j = 0; j < QF; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, kr[u][j][i]), qf[j][i], s[u], 0, 0, 0);
          } else {
            auto add = [&](int j, au32x4_t k) {
              const bf16x8_t kb = as_frag(k);
#pragma unroll
              for (int q = F::kQTerms - 1; q >= 0; --q) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qb[q][j], s[u], 0, 0, 0);
            };
#pragma unroll
            for (int j = 0; j < F::kKLoads; ++j) {
              if constexpr (TYPE == KC_INT8) {
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                  float x[4], y[4];
                  int8_to_floats(kr[u][j][2 * w], x);
                  int8_to_floats(kr[u][j][2 * w + 1], y);
                  add(2 * j + w, au32x4_t{top_halves(x[0], x[1]), top_halves(x[2], x[3]), top_halves(y[0], y[1]), top_halves(y[2], y[3])});
                }
              } else if constexpr (TYPE == KC_E4M3) {
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                  const uint32_t x = kr[u][j][2 * w], y = kr[u][j][2 * w + 1];
                  add(2 * j + w, au32x4_t{e4m3_to_bf16<false>(x), e4m3_to_bf16<true>(x), e4m3_to_bf16<false>(y), e4m3_to_bf16<true>(y)});
                }
              } else {
                add(j, au32x4_t{kr[u][j][0], kr[u][j][1], kr[u][j][2], kr[u][j][3]});
              }
            }
          }
        }
        // scores ahead of their scale
        float p[NT][4];
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[u][i] = s[u][i];
            if constexpr (F::kCoded) p[u][i] *= ks[u][i];
          }
        // a step that not all rows see all of
        bool part = pos < all_lo || pos + STEP - 1 > all_hi;
#pragma unroll
        for (int u = 0; u < NT; ++u) part |= k_valid[u] < kKvTile;
        uint32_t seen = 0xff;             // bit u * 4 + i
        if (part) {
          seen = 0;
#pragma unroll
          for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int32_t x = pos + u * kKvTile + 4 * g + i;
              const bool in = x >= lo && x <= hi && 4 * g + i < k_valid[u];
              seen |= (uint32_t)in << (u * 4 + i);
              if (!in) p[u][i] = -INFINITY;
              if constexpr (F::kCoded) vs[u][i] = in ? vs[u][i] : 0.f;   // (the scale of a place that holds nothing may be anything)
            }
        }
        // the next step's keys, into the registers that have been read
        int32_t id_cur[NT];
#pragma unroll
        for (int u = 0; u < NT; ++u) id_cur[u] = id_next[u];
        load_k(pos + stride, id_cur);
#pragma unroll
        for (int u = 0; u < NT; ++u) id_next[u] = page_of(pos + 2 * stride + u * kKvTile);

        float top = p[0][0];
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, p[u][i]);
        // The maximum that weights are relative to may lag behind the true one by a factor of 2^8, which floats do not mind: it moves less often.
        // It is held ahead of the scale, which the difference is multiplied with: 0 where a score is the maximum, whatever its size (that of
        // scaled ones is a rounding error, past the exponential's range from 2^31 on).
        const float seen_top = max_of_rows(top);
        if (__any((seen_top - m) * a.scale_log2 > 8.f)) {
          const float m_new = fmaxf(m, seen_top), f = __builtin_amdgcn_exp2f((m - m_new) * a.scale_log2);   // (seen_top > -inf somewhere: other rows may have none yet)
          const float by = m_new == -INFINITY ? 1.f : f;
          l *= by;
#pragma unroll
          for (int j = 0; j < NO; ++j) o[j] *= by;
          m = m_new;
        }
        const float m_use = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[u][i] = __builtin_amdgcn_exp2f((p[u][i] - m_use) * a.scale_log2);
            l += p[u][i];
            if constexpr (F::kCoded) p[u][i] *= vs[u][i];
          }
        // Values that only some rows see must not reach the others, whatever they are: 0 times an infinity or a NaN is a NaN.  Such values
        // are taken out, and the columns of the rows that see them made NaN.
        if constexpr (F::kCanBeOdd) {
          uint32_t odd = 0;
          if (part) {
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < F::kVHalves; ++h)
#pragma unroll
                  for (int w = 0; w < F::kVDwords; ++w) {
                    uint32_t x = vr[u][i][h][w];
                    asm volatile("" : "+v"(x));   // (or the compiler does this in every step, ahead of the branch)
                    odd |= F::odd(x);
                  }
          }
          if (__any(odd != 0)) {
            auto ones = [&](int u, int i, int h, int w) { return F::odd_bits(vr[u][i][h][w]) & F::kOnes; };
            if constexpr (F::kF32) {
              f32x4_t count;
              columns(ones, [&](int j, int i, float x) {
                if (i == 0) count = f32x4_t{};
                count = __builtin_amdgcn_mfma_f32_16x16x4f32(x, seen >> i & 1 ? 1.f : 0.f, count, 0, 0, 0);
                if (i == 3)
#pragma unroll
                  for (int r = 0; r < 4; ++r) o[j][r] = count[r] > 0.f ? __builtin_nanf("") : o[j][r];
              });
            } else {
              bf16x8_t sb;
#pragma unroll
              for (int k = 0; k < 8; ++k) sb[k] = (bf16_t)(seen >> k & 1 ? 1.f : 0.f);
              columns(ones, [&](int j, bf16x8_t x) {
                const f32x4_t count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, sb, f32x4_t{}, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[j][r] = count[r] > 0.f ? __builtin_nanf("") : o[j][r];
              });
            }
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < F::kVHalves; ++h)
#pragma unroll
                  for (int w = 0; w < F::kVDwords; ++w) vr[u][i][h][w] &= ~F::odd_bits(vr[u][i][h][w]);
          }
        }
        auto as_loaded = [&](int u, int i, int h, int w) { return vr[u][i][h][w]; };
        if constexpr (F::kF32) {
          columns(as_loaded, [&](int j, int i, float x) { o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, p[0][i], o[j], 0, 0, 0); });
        } else {
          bf16x8_t pb[F::kPTerms];
          float rest[8];
#pragma unroll
          for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) rest[u * 4 + i] = p[u][i];
#pragma unroll
          for (int s = 0; s < F::kPTerms; ++s) {
            au32x4_t term;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t two = pack_bf16(rest[2 * k], rest[2 * k + 1]);
              term[k] = two;
              rest[2 * k] -= lo_bf16(two);
              rest[2 * k + 1] -= hi_bf16(two);
            }
            pb[s] = as_frag(term);
          }
          columns(as_loaded, [&](int j, bf16x8_t vb) {
#pragma unroll
            for (int s = 0; s < F::kPTerms; ++s) o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, pb[s], o[j], 0, 0, 0);
          });
        }
        load_v();
      }
    }

    // ---- the waves' parts
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    __syncthreads();                      // (the last segment's have been read)
    float* own = lds + wave * 16 * LD;
#pragma unroll
    for (int h = 0; h < F::kVHalves; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < F::kVW; e += 4)
          *reinterpret_cast<f32x4_t*>(own + c * LD + (h * 16 + g * 4 + i) * F::kVW + e) =
              f32x4_t{o[h * F::kVW + e][i], o[h * F::kVW + e + 1][i], o[h * F::kVW + e + 2][i], o[h * F::kVW + e + 3][i]};
    if (g == 0) {
      lds_ml[(wave * 16 + c) * 2] = m;
      lds_ml[(wave * 16 + c) * 2 + 1] = l;
    }
    __syncthreads();
    const int64_t slot = 2 * (int64_t)blockIdx.x + (chunk == 0);
    const int quads = a.D / 4, rows_here = a.R - group * a.group_rows < a.group_rows ? a.R - group * a.group_rows : a.group_rows;
    for (int x = threadIdx.x; x < rows_here * quads; x += WAVES * 64) {
      const int r = kv_div(x, a.by_quads), d = (x - r * quads) * 4, tile = r >> 4, r16 = r & 15;
      // (all waves' at once: those of other tiles of rows do not count, whatever they are)
      float ms[WAVES], ls[WAVES];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        ms[w] = lds_ml[(w * 16 + r16) * 2];
        ls[w] = lds_ml[(w * 16 + r16) * 2 + 1];
      }
      bool ours[WAVES];
#pragma unroll
      for (int w = 0, of = 0; w < WAVES; ++w) {
        ours[w] = of == tile;
        if (!ours[w]) ms[w] = -INFINITY;
        of = of + 1 == a.tile_waves ? 0 : of + 1;
      }
      float top = ms[0], sum = 0.f;
#pragma unroll
      for (int w = 1; w < WAVES; ++w) top = fmaxf(top, ms[w]);
      const float use = top == -INFINITY ? 0.f : top;
      f32x4_t v = {};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f((ms[w] - use) * a.scale_log2);
        const f32x4_t part = *reinterpret_cast<const f32x4_t*>(lds + (w * 16 + r16) * LD + d);
        if (ours[w]) {
          sum += f * ls[w];
          v += f * part;
        }
      }
      const int rr = group * a.group_rows + r;
      if (whole) {
        const int tt = a.T == 1 ? 0 : rr / a.G;
        const int64_t o_row = ((int64_t)b * a.T + tt) * (a.heads * a.G) + head * a.G + (rr - tt * a.G);
        const bool some = sum != 0.f;     // (NaN: some)
        const float inv = 1.f / sum;
        if (!some) v = f32x4_t{};
        else v *= inv;
        if constexpr (F32Q) *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + o_row * a.D + d) = v;
        else *reinterpret_cast<au32x2_t*>(reinterpret_cast<uint16_t*>(a.out) + o_row * a.D + d) = au32x2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        if (d == 0 && a.lse) a.lse[o_row] = some ? top * a.scale + logf(sum) : -INFINITY;
      } else {
        *reinterpret_cast<f32x4_t*>(a.part + (slot * a.group_rows + r) * a.D + d) = v;
        if (d == 0) {
          a.part_ml[(slot * a.group_rows + r) * 2] = top;
          a.part_ml[(slot * a.group_rows + r) * 2 + 1] = sum;
        }
      }
    }
    // on to what comes next in the run
    left -= here;
    chunk = 0;
    if (left > 0 && ++hr == a.heads * a.row_groups) {
      hr = 0;
      do ++b;
      while (seq_span(a, b).chunks == 0);   // (there is one: chunks are left)
    }
  } while (left > 0);
}

// ---- parts of several blocks -------------------------------------------------------
// A row of a (sequence, head, row group) joined by a block, its row by blockIdx.y.  Which one: by blockIdx.x, or, where there are more of them
// than runs (by_runs), the one inside of which run blockIdx.x begins: few are shared then.  Groups of D / 4 lanes (a power of two of
// them) take the parts in turns; the order of the sums is that of the parts and the groups.
// us, the whole call, by number / by run: 1024 sequences up to 2048 tokens, 8 heads of 128 in bf16 803 / 767; 4096 up to 1100, 8 of 64 in int8
// 1160 / 632.
template <bool F32Q, int WAVES> __global__ __launch_bounds__(WAVES * 64) void kv_join_kernel(KvAttnDev a, int blocks, int lanes_log, bool by_runs) {
  constexpr int THREADS = WAVES * 64;
  __shared__ int32_t s_sum[WAVES], s_found[2];
  __shared__ f32x2_t s_l[THREADS];
  __shared__ f32x4_t s_o[THREADS];
  const int hrs = a.heads * a.row_groups, r = blockIdx.y;
  int b, hr;
  int32_t k0 = 0, parts = 0;              // the first block that has some of it, and how many
  auto store = [&](int b, int hr, int d, f32x4_t v, float lse) {
    const int head = hr / a.row_groups, rr = (hr - head * a.row_groups) * a.group_rows + r, t = a.T == 1 ? 0 : rr / a.G;
    const int64_t o_row = ((int64_t)b * a.T + t) * (a.heads * a.G) + head * a.G + (rr - t * a.G);
    if constexpr (F32Q) *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + o_row * a.D + d) = v;
    else *reinterpret_cast<au32x2_t*>(reinterpret_cast<uint16_t*>(a.out) + o_row * a.D + d) = au32x2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    if (d == 0 && a.lse) a.lse[o_row] = lse;
  };
  auto row_there = [&](int hr) { return hr % a.row_groups * a.group_rows + r < a.R; };
  if (by_runs) {
    // those of sequences that hold nothing no run has: a lane each
    for (int64_t x = (int64_t)blockIdx.x * THREADS + threadIdx.x; x < (int64_t)a.B * hrs; x += (int64_t)blocks * THREADS) {
      const int eb = (int)x / hrs, ehr = (int)x - eb * hrs;
      if (!row_there(ehr) || seq_span(a, eb).chunks > 0) continue;
      for (int d = 0; d < a.D; d += 4) store(eb, ehr, d, f32x4_t{}, -INFINITY);
    }
    const Run run = cut_run<WAVES>(a, s_sum, s_found);
    if (run.left <= 0 || run.chunk == 0 || !row_there(run.hr)) return;
    b = run.b;
    hr = run.hr;
    const int32_t at = (int32_t)blockIdx.x * run.per - run.chunk;
    k0 = at / run.per;
    if (k0 + 1 != (int32_t)blockIdx.x) return;   // an earlier run begins in it too
    parts = (at + seq_span(a, b).chunks - 1) / run.per - k0 + 1;
  } else {
    b = blockIdx.x / hrs;
    hr = blockIdx.x - b * hrs;
    if (!row_there(hr)) return;
    const SeqSpan span = seq_span(a, b);
    if (span.chunks > 0) {
      Cut cut;
      int32_t ahead;                      // units of the sequences ahead
      if (a.B <= 64) {
        const LaneCut l = cut_lanes(a, blocks);
        cut = l.cut;
        ahead = __builtin_amdgcn_readlane(l.ahead, b);
      } else {
        cut = cut_all<WAVES>(a, blocks, s_sum);
        int32_t n = 0;
        for (int i = threadIdx.x; i < b; i += THREADS) n += cut.units(seq_span(a, i).chunks);
        ahead = sum_of_waves<WAVES>(n, s_sum) * hrs;
      }
      const int32_t units = cut.units(span.chunks), at = ahead + hr * units;
      k0 = cut.pieces ? at : at / cut.per;
      parts = cut.pieces ? units : (at + units - 1) / cut.per - k0 + 1;
      if (parts == 1) return;             // one block's, written by it
    }
  }
  // part k of the pair: its block's slot 2 blk + 1 where the pair begins, else 2 blk
  auto slot = [&](int32_t k) { return (2 * (int64_t)(k0 + k) + (k == 0)) * a.group_rows + r; };
  const int groups = THREADS >> lanes_log, gr = threadIdx.x >> lanes_log, d = (threadIdx.x & ((1 << lanes_log) - 1)) * 4;
  float top = -INFINITY, sum = 0.f;       // a group's, with its running maximum: one wait for the loads of all its parts
  f32x4_t v = {};
#pragma unroll 4
  for (int32_t k = gr; k < parts; k += groups) {
    const int64_t s = slot(k);
    const f32x2_t ml = *reinterpret_cast<const f32x2_t*>(a.part_ml + s * 2);
    f32x4_t part = {};
    if (d < a.D) part = *reinterpret_cast<const f32x4_t*>(a.part + s * a.D + d);
    const float m = fmaxf(top, ml[0]), use = m == -INFINITY ? 0.f : m;
    const float f = __builtin_amdgcn_exp2f((top - use) * a.scale_log2), by = __builtin_amdgcn_exp2f((ml[0] - use) * a.scale_log2);
    sum = sum * f + by * ml[1];
    v = v * f + by * part;
    top = m;
  }
  s_o[threadIdx.x] = v;
  s_l[threadIdx.x] = f32x2_t{top, sum};
  __syncthreads();
  if (gr != 0) return;
  for (int x = 1; x < groups; ++x) top = fmaxf(top, s_l[(x << lanes_log) + threadIdx.x][0]);
  const float use = top == -INFINITY ? 0.f : top;
  v = f32x4_t{};
  sum = 0.f;
  for (int x = 0; x < groups; ++x) {
    const f32x2_t ml = s_l[(x << lanes_log) + threadIdx.x];
    const float by = __builtin_amdgcn_exp2f((ml[0] - use) * a.scale_log2);
    sum += by * ml[1];
    v += by * s_o[(x << lanes_log) + threadIdx.x];
  }
  const bool some = sum != 0.f;           // (NaN: some)
  if (!some) v = f32x4_t{};
  else v *= 1.f / sum;
  if (d < a.D) store(b, hr, d, v, some ? top * a.scale + logf(sum) : -INFINITY);
}

// ---- host --------------------------------------------------------------------------
struct AttnPlan {
  int G, R, row_tiles, tile_waves, row_groups, group_rows;
  bool split;
  int waves, chunk, blocks;
  size_t part_ml, total;
};

as_status check_attn(const kc_cache* c, const kc_attn* s) {
  if (!s) return set_error(AS_ERR_NULL, "attn is NULL");
  if (s->T < 1 || s->T > 64 || s->q_heads < 1 || s->q_heads % c->heads != 0 || (int64_t)s->T * (s->q_heads / c->heads) > 1024)
    return set_error(AS_ERR_SHAPE, "%d tokens of %d heads of queries, %d of the cache", s->T, s->q_heads, c->heads);
  if (s->max_len < 1 || s->max_len > (int64_t)c->max_pages * c->page || s->max_len >= 1 << 28)
    return set_error(AS_ERR_SHAPE, "max_len=%d with %d pages of %d tokens to a sequence", s->max_len, c->max_pages, c->page);
  if (s->window < 0 || !std::isfinite(s->scale * kLog2e)) return set_error(AS_ERR_SHAPE, "window=%d scale=%g", s->window, (double)s->scale);
  const int64_t pairs = (int64_t)c->B * c->heads * ((s->T * (s->q_heads / c->heads) + 63) / 64);
  // a launch takes less than 2^32 threads along a dimension, and chunks are counted in 31 bits
  if (pairs > 1 << 22 || pairs * ((s->max_len + kLeastChunk - 1) / kLeastChunk + 1) >= (int64_t)1 << 30)
    return set_error(AS_ERR_SHAPE, "%d sequences of %d heads up to %d tokens are too many for one call", c->B, c->heads, s->max_len);
  return AS_OK;
}

AttnPlan attn_plan(const kc_cache* c, const kc_attn* s) {
  AttnPlan p;
  p.G = s->q_heads / c->heads;
  p.R = s->T * p.G;
  p.row_tiles = (p.R + 15) / 16;
  p.tile_waves = p.row_tiles < 4 ? p.row_tiles : 4;
  p.row_groups = (p.row_tiles + p.tile_waves - 1) / p.tile_waves;
  p.group_rows = p.row_groups > 1 ? p.tile_waves * 16 : p.R;
  int64_t span = s->max_len;
  if (s->window > 0 && (int64_t)s->window + s->T + kKvTile < span) span = (int64_t)s->window + s->T + kKvTile;
  const int step = c->cache_type == KC_F32 ? kKvTile : 2 * kKvTile;
  const int64_t pairs = (int64_t)c->B * c->heads * p.row_groups;
  // Up to so many steps of eight waves a block takes all of a (sequence, head).
  p.split = span > (int64_t)kWholeSteps * (c->D > 128 ? 4 : 8) / p.tile_waves * step;
  // Four waves to a block: twice as many blocks, so that one's beginning and end are the other's middle.  Eight where few blocks are all
  // there are, and for three and four tiles of rows, whose waves share tokens.  us, 8 / 4: 64 sequences up to 8192 tokens, 32 heads on 8 of 128,
  // bf16 210 / 205, e4m3 141 / 123; 256 up to 300 74 / 44; one of 700, 8 heads of 64 10.5 / 13.2; 24 of 1004 tokens seen by 40 rows 22 / 25.
  p.waves = c->D > 128 ? 4 : p.tile_waves >= 3 || (!p.split && pairs < 512) ? 8 : 4;
  p.chunk = p.waves / p.tile_waves * step;   // a step of every wave
  const int64_t chunks = (span + p.chunk - 1) / p.chunk;
  int64_t blocks = pairs;
  if (p.split) {
    blocks = pairs * chunks;
    // what the compute units hold
    const int64_t most = c->D > 128 ? 256 : (c->D <= 64 ? 4096 : 2048) / p.waves;
    if (blocks > most) blocks = most;
  }
  p.blocks = (int)blocks;
  const size_t rows = p.split ? (size_t)2 * p.blocks * p.group_rows : 0;
  p.part_ml = (rows * c->D * 4 + 255) / 256 * 256;
  p.total = p.part_ml + rows * 8;
  if (p.total < 16) p.total = 16;
  return p;
}

template <int TYPE, bool F32Q, int DP, int WAVES> hipError_t launch_attn(const KvAttnDev& a, dim3 blocks, hipStream_t st) {
  constexpr int smem = WAVES * 16 * (DP + 4 + 2) * 4;
  auto kfn = kv_attn_kernel<TYPE, F32Q, DP, WAVES>;
  static LdsLimit limit;
  const hipError_t e = limit.raise(reinterpret_cast<const void*>(kfn), smem);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kfn, blocks, dim3(WAVES * 64), smem, st, a);
  return hipGetLastError();
}
template <int TYPE, bool F32Q> hipError_t launch_attn_any(const KvAttnDev& a, const AttnPlan& p, hipStream_t st) {
  const dim3 blocks = p.split ? dim3(p.blocks) : dim3(a.B, a.heads * a.row_groups);
  if (a.D > 128) return launch_attn<TYPE, F32Q, 256, 4>(a, blocks, st);
  if (a.D > 64) return p.waves == 8 ? launch_attn<TYPE, F32Q, 128, 8>(a, blocks, st) : launch_attn<TYPE, F32Q, 128, 4>(a, blocks, st);
  return p.waves == 8 ? launch_attn<TYPE, F32Q, 64, 8>(a, blocks, st) : launch_attn<TYPE, F32Q, 64, 4>(a, blocks, st);
}

}  // namespace
}  // namespace asx

using namespace asx;

extern "C" size_t kv_cache_attn_workspace_bytes(const kc_cache* cache, const kc_attn* attn) {
  if (kv_check_cache(cache) != AS_OK || check_attn(cache, attn) != AS_OK) return 0;
  return attn_plan(cache, attn).total;
}

extern "C" as_status kv_cache_attn(const kc_cache* cache, const kc_attn* attn, const void* q, int64_t ld_q, const void* k_pages,
                                   const void* v_pages, const float* k_scales, const float* v_scales, const int32_t* page_table,
                                   const int32_t* lengths, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  as_status rc = kv_check_cache(cache);
  if (rc == AS_OK) rc = check_attn(cache, attn);
  if (rc != AS_OK) return rc;
  if (!q || !lengths || !out || !workspace) return set_error(AS_ERR_NULL, "kv_cache_attn: a required pointer is NULL");
  rc = kv_check_pool(cache, k_pages, v_pages, k_scales, v_scales, page_table, "kv_cache_attn");
  if (rc != AS_OK) return rc;
  const bool f32 = cache->dtype == AS_F32;
  if (ld_q < (int64_t)attn->q_heads * cache->D || ld_q >= (int64_t)1 << 32) return set_error(AS_ERR_SHAPE, "kv_cache_attn: rows %lld elements apart", (long long)ld_q);
  if (ld_q * (f32 ? 4 : 2) % 16 != 0) return set_error(AS_ERR_ALIGN, "kv_cache_attn: rows %lld elements apart do not start on 16 bytes", (long long)ld_q);
  const AttnPlan p = attn_plan(cache, attn);
  if (workspace_bytes < p.total) return set_error(AS_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, p.total);
  for (const void* x : {q, (const void*)lengths, (const void*)out, (const void*)lse, (const void*)workspace})
    if (!kv_al16(x)) return set_error(AS_ERR_ALIGN, "kv_cache_attn: a pointer is not 16-byte aligned");
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  KvAttnDev a;
  a.q = q;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.table = page_table;
  a.lengths = lengths;
  a.out = out;
  a.lse = lse;
  a.part = reinterpret_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float*>(ws + p.part_ml);
  a.ld_q = ld_q;
  a.B = cache->B;
  a.T = attn->T;
  a.heads = cache->heads;
  a.G = p.G;
  a.D = cache->D;
  a.R = p.R;
  a.tile_waves = p.tile_waves;
  a.tok_waves = p.waves / p.tile_waves;
  a.by_tile_waves = kv_magic((uint32_t)p.tile_waves);
  a.by_quads = kv_magic((uint32_t)cache->D / 4);
  a.row_groups = p.row_groups;
  a.group_rows = p.group_rows;
  a.page = cache->page;
  a.page_tiles = cache->page / kKvTile;
  a.pages = cache->pages;
  a.max_pages = cache->max_pages;
  a.max_len = attn->max_len;
  a.window = attn->window < attn->max_len ? attn->window : 0;   // (longer ones are none)
  a.magic = kv_magic((uint32_t)a.page_tiles);
  a.chunk = p.chunk;
  a.split = p.split;
  // (of scale 0 the queries are read as 0: masked scores are -inf, whose product with 0 would be none)
  a.scale = std::fabs(attn->scale);
  a.scale_log2 = attn->scale != 0.f ? std::fabs(attn->scale) * kLog2e : 1.f;
  a.no_q = attn->scale == 0.f;
  a.q_sign = attn->scale < 0 ? f32 ? 0x80000000u : 0x80008000u : 0u;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  hipError_t e;
  switch (cache->cache_type) {
    case KC_F32: e = launch_attn_any<KC_F32, true>(a, p, st); break;
    case KC_BF16: e = launch_attn_any<KC_BF16, false>(a, p, st); break;
    case KC_INT8: e = f32 ? launch_attn_any<KC_INT8, true>(a, p, st) : launch_attn_any<KC_INT8, false>(a, p, st); break;
    default: e = f32 ? launch_attn_any<KC_E4M3, true>(a, p, st) : launch_attn_any<KC_E4M3, false>(a, p, st); break;
  }
  if (e == hipSuccess && p.split) {
    const int64_t pairs = (int64_t)cache->B * cache->heads * p.row_groups;
    const bool by_runs = pairs > p.blocks;      // (runs they are then, not pieces)
    const dim3 grid((unsigned)(by_runs ? p.blocks : pairs), (unsigned)p.group_rows);
    int lanes_log = 2;
    while (4 << lanes_log < cache->D) ++lanes_log;
    // many parts, or many sequences to look through: four waves to a row (256 sequences, one wave / four: 80 / 85 us)
    const bool many = by_runs ? cache->B > 1024 : p.blocks > 8 * pairs;
    auto kfn = f32 ? many ? kv_join_kernel<true, 4> : kv_join_kernel<true, 1> : many ? kv_join_kernel<false, 4> : kv_join_kernel<false, 1>;
    hipLaunchKernelGGL(kfn, grid, dim3(many ? 256 : 64), 0, st, a, p.blocks, lanes_log, by_runs);
    e = hipGetLastError();
  }
  return e == hipSuccess ? AS_OK : set_error(AS_ERR_HIP, "kv_cache_attn: %s", hipGetErrorString(e));
}
