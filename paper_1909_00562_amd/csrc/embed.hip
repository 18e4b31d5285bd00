// Embedding lookup with scaling, and its gradient by sorted words (entry points and kernels).
//
// Forward: a row copy with a multiplication; bound by memory.
// Backward: d_table[v] = scale * sum of dy[n] over the positions n of word v.  Words are Zipf-like: one word has a tenth of all
// positions, most have none.  The positions are sorted by word (stable radix sort, so each word's rows are added in increasing
// n, whatever the launch looks like: no float atomics), the sorted list is cut into pieces of the same length, and a group of
// threads adds up the rows of its piece, whatever words they are of.  Words that lie inside a piece are written at once; parts
// of words that reach over a piece's edge go to the workspace, and a second pass adds those up.  Rows of words that no position has
// are zeroed by further blocks of the same launch, by a bitmap that the sort leaves: d_table is written once.
#include "../../include/vocab_ops.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "common.h"
#include "lds_limit.h"
#include "status.h"

namespace asx {
namespace {

typedef uint32_t eu32x4_t __attribute__((ext_vector_type(4)));

// Elements a thread moves at a time (16 bytes, or one where rows do not start on 16 bytes), as floats.
template <typename TE, int VEC> __device__ __forceinline__ void ld_vec(const TE* p, float (&f)[VEC]) {
  if constexpr (VEC == 1) {
    f[0] = ld_elem<TE>(p, 0);
  } else {
    const eu32x4_t q = *reinterpret_cast<const eu32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(TE) == 2) {
        f[2 * i] = lo_bf16(q[i]);
        f[2 * i + 1] = hi_bf16(q[i]);
      } else {
        const uint32_t w = q[i];   // (a bit cast of the vector's element itself reads element 0)
        f[i] = __builtin_bit_cast(float, w);
      }
    }
  }
}
template <typename TE, int VEC> __device__ __forceinline__ void st_vec(TE* p, const float (&f)[VEC]) {
  if constexpr (VEC == 1) {
    st_elem<TE>(p, 0, f[0]);
  } else {
    eu32x4_t q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = sizeof(TE) == 2 ? pack_bf16(f[VEC / 4 * i], f[VEC / 4 * i + VEC / 4 - 1]) : __builtin_bit_cast(uint32_t, f[i]);
    *reinterpret_cast<eu32x4_t*>(p) = q;
  }
}

// the word of position n, V at padding (sorts behind all words)
__device__ __forceinline__ uint32_t word_key(const int32_t* ids, int n, int V, int pad_id) {
  const int id = ids[n];
  return id >= 0 && id < V && id != pad_id ? (uint32_t)id : (uint32_t)V;
}

// ---- forward -----------------------------------------------------------------------
// 2^tpr_log threads per row
template <typename TE, int VEC>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const TE* __restrict__ table, const int32_t* __restrict__ ids, int N,
                                                        int I, int V, int pad_id, float scale, TE* __restrict__ x, int tpr_log) {
  const int64_t n = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> tpr_log;
  if (n >= N) return;
  const int lane = threadIdx.x & ((1 << tpr_log) - 1), step = VEC << tpr_log;
  const uint32_t w = word_key(ids, (int)n, V, pad_id);
  TE* out = x + n * I;
  const TE* row = table + (int64_t)(w < (uint32_t)V ? w : 0) * I;
  for (int c = lane * VEC; c < I; c += step) {
    float f[VEC];
    if (w < (uint32_t)V) {
      ld_vec<TE, VEC>(row + c, f);
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] *= scale;
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] = 0.f;
    }
    st_vec<TE, VEC>(out + c, f);
  }
}

// ---- the sort ----------------------------------------------------------------------
// Stable radix sort of (word, position) by digits of up to 9 bits.  A wave owns a contiguous run of the keys and walks it 64 at a
// time: lanes with the same digit find each other by ballots, their rank is the number of lower such lanes, the wave's
// running count of the digit is in its own row of LDS.  Digits' places: all counts of lower digits, then those of earlier
// waves (and blocks).
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kDigitBits = 9;
constexpr int kSortOne = 8192;   // keys that one block sorts in LDS

__device__ __forceinline__ uint64_t same_digit(uint32_t d, int bits, uint64_t in) {
  uint64_t m = in;
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((d >> b) & 1u);
    m &= (d >> b) & 1u ? set : ~set;
  }
  return m;
}
__device__ __forceinline__ void lds_in_order() {   // this wave's LDS accesses before it are done before those behind it
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// count[wave][digit] of the keys [beg, end) of this wave
template <typename Key>
__device__ __forceinline__ void count_digits(Key key, int beg, int end, int shift, int bits, uint32_t* row) {
  const int lane = threadIdx.x & 63;
  for (int d = lane; d < 1 << bits; d += 64) row[d] = 0;
  lds_in_order();
  for (int i0 = beg; i0 < end; i0 += 64) {
    const bool in = i0 + lane < end;
    const uint32_t d = in ? (key(i0 + lane) >> shift) & ((1u << bits) - 1) : 0;
    const uint64_t m = same_digit(d, bits, __ballot(in));
    if (in && (m & ((1ull << lane) - 1)) == 0) row[d] += __popcll(m);
    lds_in_order();
  }
}
// put(place, i) for the keys [beg, end); row: the places of the wave's first key of each digit
template <typename Key, typename Put>
__device__ __forceinline__ void place_digits(Key key, Put put, int beg, int end, int shift, int bits, uint32_t* row) {
  const int lane = threadIdx.x & 63;
  for (int i0 = beg; i0 < end; i0 += 64) {
    const bool in = i0 + lane < end;
    const uint32_t k = in ? key(i0 + lane) : 0, d = (k >> shift) & ((1u << bits) - 1);
    const uint64_t m = same_digit(d, bits, __ballot(in));
    const int rank = __popcll(m & ((1ull << lane) - 1));
    const uint32_t at = row[d] + rank;
    lds_in_order();
    if (in) put(at, i0 + lane, k);
    if (in && rank == 0) row[d] += __popcll(m);
    lds_in_order();
  }
}
// exclusive prefix of one value per thread over the block; *total: the sum
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, uint32_t* waves, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t t = __shfl_up(s, o, 64);
    if (lane >= o) s += t;
  }
  if (lane == 63) waves[wave] = s;
  __syncthreads();
  uint32_t base = 0, sum = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    if (w < wave) base += waves[w];
    sum += waves[w];
  }
  __syncthreads();
  *total = sum;
  return base + s - v;
}
// counts [wave][digit] of one block -> places, digit-major; base: where digit d of this block begins (or null: from 0 on)
__device__ __forceinline__ void digit_places(uint32_t* count, int bits, const uint32_t* base, int64_t base_step, uint32_t* waves) {
  const int bins = 1 << bits;
  uint32_t carry = 0;
  for (int d0 = 0; d0 < bins; d0 += kSortThreads) {
    const int d = d0 + threadIdx.x;
    uint32_t sum = 0, total;
    if (d < bins)
      for (int w = 0; w < kSortWaves; ++w) sum += count[w * bins + d];
    uint32_t at = carry + block_prefix(sum, waves, &total);
    carry += total;
    if (d < bins) {
      if (base) at = base[d * base_step];
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = count[w * bins + d];
        count[w * bins + d] = at;
        at += c;
      }
    }
  }
  __syncthreads();
}

struct SortDev {
  const int32_t* ids;
  int N, V, pad_id;
  int passes, bits;         // digits and their bits
  uint32_t *key, *pos;      // the sorted words and positions
  uint32_t* bitmap;         // a bit per word: some position has it
  int bitmap_words;
};

// N <= kSortOne: one block, keys and positions in LDS
__global__ __launch_bounds__(kSortThreads) void sort_one_kernel(SortDev p) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int N = p.N, bins = 1 << p.bits, tid = threadIdx.x, wave = tid >> 6;
  const int N64 = (N + 63) & ~63;
  uint32_t* k0 = reinterpret_cast<uint32_t*>(smem);
  uint32_t* k1 = k0 + N64;
  uint32_t* count = k1 + N64;
  uint32_t* waves = count + kSortWaves * bins;
  uint16_t* p0 = reinterpret_cast<uint16_t*>(waves + kSortWaves);
  uint16_t* p1 = p0 + N64;
  for (int i = tid; i < p.bitmap_words; i += kSortThreads) p.bitmap[i] = 0;
  for (int i = tid; i < N; i += kSortThreads) {
    k0[i] = word_key(p.ids, i, p.V, p.pad_id);
    p0[i] = (uint16_t)i;
  }
  __threadfence();   // the bitmap's zeros, ahead of the bits below
  __syncthreads();
  const int per = ((N + kSortWaves - 1) / kSortWaves + 63) & ~63;
  const int beg = wave * per < N ? wave * per : N, end = beg + per < N ? beg + per : N;
  for (int d = 0; d < p.passes; ++d) {
    count_digits([&](int i) { return k0[i]; }, beg, end, d * p.bits, p.bits, count + wave * bins);
    __syncthreads();
    digit_places(count, p.bits, nullptr, 0, waves);
    place_digits([&](int i) { return k0[i]; },
                 [&](uint32_t at, int i, uint32_t k) {
                   k1[at] = k;
                   p1[at] = p0[i];
                 },
                 beg, end, d * p.bits, p.bits, count + wave * bins);
    __syncthreads();
    uint32_t* tk = k0; k0 = k1; k1 = tk;
    uint16_t* tp = p0; p0 = p1; p1 = tp;
  }
  for (int i = tid; i < N; i += kSortThreads) {
    const uint32_t k = k0[i];
    p.key[i] = k;
    p.pos[i] = p0[i];
    if (k < (uint32_t)p.V && (i == 0 || k0[i - 1] != k)) atomicOr(p.bitmap + (k >> 5), 1u << (k & 31));
  }
}

// More keys: per digit a count, the places of all digits of all blocks, and the move.  A block's waves own runs of `per` keys.
struct SortPass {
  const uint32_t *key_in, *pos_in;   // null: the first pass, from the ids
  uint32_t *key_out, *pos_out;
  uint32_t* places;                  // [digit][block]
  int blocks, per, shift;
};
__device__ __forceinline__ uint32_t pass_key(const SortDev& p, const SortPass& s, int i) {
  return s.key_in ? s.key_in[i] : word_key(p.ids, i, p.V, p.pad_id);
}
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortDev p, SortPass s) {
  __shared__ uint32_t count[kSortWaves << kDigitBits];
  const int bins = 1 << p.bits, wave = threadIdx.x >> 6;
  const int64_t b0 = ((int64_t)blockIdx.x * kSortWaves + wave) * s.per;
  const int beg = b0 < p.N ? (int)b0 : p.N, end = b0 + s.per < p.N ? (int)(b0 + s.per) : p.N;
  count_digits([&](int i) { return pass_key(p, s, i); }, beg, end, s.shift, p.bits, count + wave * bins);
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += kSortThreads) {
    uint32_t sum = 0;
    for (int w = 0; w < kSortWaves; ++w) sum += count[w * bins + d];
    s.places[(int64_t)d * s.blocks + blockIdx.x] = sum;
  }
}
__global__ __launch_bounds__(kSortThreads) void sort_places_kernel(SortDev p, SortPass s) {
  __shared__ uint32_t waves[kSortWaves];
  if (!s.key_in)
    for (int i = threadIdx.x; i < p.bitmap_words; i += kSortThreads) p.bitmap[i] = 0;
  const int total = s.blocks << p.bits;   // <= 2^18
  const int per = (total + kSortThreads - 1) / kSortThreads, beg = threadIdx.x * per;
  uint32_t sum = 0, all;
  for (int i = beg; i < beg + per && i < total; ++i) sum += s.places[i];
  uint32_t at = block_prefix(sum, waves, &all);
  for (int i = beg; i < beg + per && i < total; ++i) {
    const uint32_t c = s.places[i];
    s.places[i] = at;
    at += c;
  }
}
__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(SortDev p, SortPass s) {
  __shared__ uint32_t count[kSortWaves << kDigitBits];
  __shared__ uint32_t waves[kSortWaves];
  const int bins = 1 << p.bits, wave = threadIdx.x >> 6;
  const int64_t b0 = ((int64_t)blockIdx.x * kSortWaves + wave) * s.per;
  const int beg = b0 < p.N ? (int)b0 : p.N, end = b0 + s.per < p.N ? (int)(b0 + s.per) : p.N;
  auto key = [&](int i) { return pass_key(p, s, i); };
  count_digits(key, beg, end, s.shift, p.bits, count + wave * bins);
  __syncthreads();
  digit_places(count, p.bits, s.places + blockIdx.x, s.blocks, waves);
  place_digits(key,
               [&](uint32_t at, int i, uint32_t k) {
                 s.key_out[at] = k;
                 s.pos_out[at] = s.key_in ? s.pos_in[i] : (uint32_t)i;
                 if (!s.key_in && k < (uint32_t)p.V) {
                   const uint32_t bit = 1u << (k & 31);
                   if (!(__hip_atomic_load(p.bitmap + (k >> 5), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & bit)) atomicOr(p.bitmap + (k >> 5), bit);
                 }
               },
               beg, end, s.shift, p.bits, count + wave * bins);
}

// ---- the sums ----------------------------------------------------------------------
struct SumsDev {
  const uint32_t *key, *pos, *bitmap;
  const void* dy;
  void* d_table;
  float* edge;       // [piece][2][I]: the part of the word a piece begins within; of the word it ends within
  int N, I, V;
  float scale;
  int accumulate;
  int piece_blocks, pieces;
  int zero_rows;     // rows a zeroing block looks at
};

// 2^tpp_log threads per piece of L sorted positions (fewer than L rows in flight per thread: RU)
template <typename TE, int VEC, int L>
__global__ __launch_bounds__(256) void embed_sums_kernel(SumsDev p, int tpp_log) {
  constexpr int RU = L < 16 ? L : 16;
  const int I = p.I, lane = threadIdx.x & ((1 << tpp_log) - 1), step = VEC << tpp_log;
  TE* table = reinterpret_cast<TE*>(p.d_table);
  if ((int)blockIdx.x >= p.piece_blocks) {   // rows of words that no position has
    const int v0 = ((int)blockIdx.x - p.piece_blocks) * p.zero_rows, rows_at_once = 256 >> tpp_log;
    const int v1 = v0 + p.zero_rows < p.V ? v0 + p.zero_rows : p.V;
    const float zero[VEC] = {};
    for (int v = v0 + (threadIdx.x >> tpp_log); v < v1; v += rows_at_once) {
      if ((p.bitmap[v >> 5] >> (v & 31)) & 1u) continue;
      for (int c = lane * VEC; c < I; c += step) st_vec<TE, VEC>(table + (int64_t)v * I + c, zero);
    }
    return;
  }
  const int piece = (int)(((int64_t)blockIdx.x * 256 + threadIdx.x) >> tpp_log);
  if (piece >= p.pieces) return;
  const int i0 = piece * L, i1 = i0 + L < p.N ? i0 + L : p.N;
  const uint32_t first = p.key[i0];
  if (first >= (uint32_t)p.V) return;   // padding from here on
  const bool begins = i0 == 0 || p.key[i0 - 1] != first;
  const uint32_t after = i1 < p.N ? p.key[i1] : (uint32_t)p.V;
  const TE* dy = reinterpret_cast<const TE*>(p.dy);
  for (int c = lane * VEC; c < I; c += step) {
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    uint32_t cur = first;
    bool whole = begins;   // the run that is being added up began in this piece
    auto flush = [&](bool ends) {
      if (whole && ends) {
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = acc[e] * p.scale;
        TE* out = table + (int64_t)cur * I + c;
        if (p.accumulate) {
          float old[VEC];
          ld_vec<TE, VEC>(out, old);
#pragma unroll
          for (int e = 0; e < VEC; ++e) f[e] += old[e];
        }
        st_vec<TE, VEC>(out, f);
      } else {
        float* out = p.edge + ((int64_t)piece * 2 + (whole ? 1 : 0)) * I + c;
#pragma unroll
        for (int e = 0; e < VEC; ++e) out[e] = acc[e];
      }
    };
#pragma unroll 1
    for (int u0 = 0; u0 < L; u0 += RU) {
      if (i0 + u0 >= i1) break;
      float x[RU][VEC];
      uint32_t k[RU];
#pragma unroll
      for (int u = 0; u < RU; ++u) {
        const int i = i0 + u0 + u;
        k[u] = i < i1 ? p.key[i] : (uint32_t)p.V;
        if (k[u] < (uint32_t)p.V) {
          ld_vec<TE, VEC>(dy + (int64_t)p.pos[i] * I + c, x[u]);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) x[u][e] = 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < RU; ++u) {   // (past the list's end: padding)
        if (k[u] != cur) {
          if (cur < (uint32_t)p.V) flush(true);
          whole = true;
          cur = k[u];
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] += x[u][e];
      }
    }
    if (cur < (uint32_t)p.V) flush(after != cur);
  }
}

// Words that reach over a piece's edge: the block of the piece such a word begins in adds the parts of the pieces behind it up,
// 64 threads' columns x 16 phases, the phases in order.
template <typename TE, int VEC, int L>
__global__ __launch_bounds__(1024) void embed_edges_kernel(SumsDev p) {
  constexpr int CV = VEC == 1 ? 1 : 4;
  __shared__ float red[16][64 * CV];
  const int piece = blockIdx.x, last = piece * L + L - 1;
  if (last + 1 >= p.N) return;
  const uint32_t word = p.key[last];
  if (word >= (uint32_t)p.V || p.key[last + 1] != word) return;
  if (piece > 0 && p.key[piece * L] == word && p.key[piece * L - 1] == word) return;   // it began further ahead
  const int col = threadIdx.x & 63, phase = threadIdx.x >> 6, I = p.I, c = (blockIdx.y * 64 + col) * CV;
  float acc[CV];
#pragma unroll
  for (int e = 0; e < CV; ++e) acc[e] = 0.f;
  if (c < I) {
    auto add = [&](int piece_, int which) {
      const float* q = p.edge + ((int64_t)piece_ * 2 + which) * I + c;
#pragma unroll
      for (int e = 0; e < CV; ++e) acc[e] += q[e];
    };
    if (phase == 0) add(piece, 1);
#pragma unroll 1
    for (int q = piece + 1 + phase; q < p.pieces && p.key[q * L] == word; q += 16) add(q, 0);
  }
#pragma unroll
  for (int e = 0; e < CV; ++e) red[phase][col * CV + e] = acc[e];
  __syncthreads();
  if (phase != 0 || c >= I) return;
#pragma unroll 1
  for (int q = 1; q < 16; ++q)
#pragma unroll
    for (int e = 0; e < CV; ++e) acc[e] += red[q][col * CV + e];
  TE* out = reinterpret_cast<TE*>(p.d_table) + (int64_t)word * I + c;
#pragma unroll
  for (int e = 0; e < CV; ++e) {
    acc[e] *= p.scale;
    if (p.accumulate) acc[e] += ld_elem<TE>(out, e);
    st_elem<TE>(out, e, acc[e]);
  }
}

// ---- host --------------------------------------------------------------------------
constexpr size_t kAlignE = 256;
size_t upe(size_t x) { return (x + kAlignE - 1) / kAlignE * kAlignE; }
int log2_up(int64_t x) {
  int b = 0;
  while (((int64_t)1 << b) < x) ++b;
  return b;
}

struct EmbedLayout {
  int L, pieces, passes, bits, blocks, per, bitmap_words;
  bool one;
  size_t key, pos, key2, pos2, places, bitmap, edge, total;
};

bool embed_ok(const vo_embed* s) {
  if (s->N < 1 || s->N > (1 << 24) || s->I < 1 || s->I > (1 << 16) || s->V < 1 || s->V > (1 << 28)) return false;
  if ((int64_t)s->V * s->I >= (int64_t)1 << 40) return false;
  return s->pad_id >= -1 && s->pad_id < s->V && std::isfinite(s->scale);
}
bool embed_types(const vo_embed* s) {
  return (s->dtype == AS_F32 && s->grad_dtype == AS_F32) ||
         (s->dtype == AS_BF16 && (s->grad_dtype == AS_F32 || s->grad_dtype == AS_BF16));
}

EmbedLayout embed_layout(const vo_embed* s) {
  EmbedLayout L;
  const int N = s->N;
  L.one = N <= kSortOne;
  const int key_bits = log2_up((int64_t)s->V + 1);   // words and the key of padding
  L.passes = (key_bits + kDigitBits - 1) / kDigitBits;
  L.bits = (key_bits + L.passes - 1) / L.passes;
  L.blocks = (N + 4095) / 4096;
  if (L.blocks > 512) L.blocks = 512;
  L.per = ((N + L.blocks - 1) / L.blocks + kSortWaves - 1) / kSortWaves;
  L.per = (L.per + 63) & ~63;
  L.L = N <= 16384 ? 16 : 32;
  L.pieces = (N + L.L - 1) / L.L;
  L.bitmap_words = (s->V + 31) / 32;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += upe(bytes);
    return o;
  };
  L.key = take((size_t)N * 4);
  L.pos = take((size_t)N * 4);
  L.bitmap = take((size_t)L.bitmap_words * 4);
  L.key2 = L.pos2 = L.places = 0;
  if (!L.one) {
    L.key2 = take((size_t)N * 4);
    L.pos2 = take((size_t)N * 4);
    L.places = take(((size_t)L.blocks << L.bits) * 4);
  }
  L.edge = take((size_t)L.pieces * 2 * s->I * 4);
  L.total = off;
  return L;
}

as_status embed_check(const vo_embed* s) {
  if (!s) return set_error(AS_ERR_NULL, "shape is NULL");
  if (!embed_types(s)) return set_error(AS_ERR_DTYPE, "vocab_embed: dtype %d with grad_dtype %d", s->dtype, s->grad_dtype);
  if (!embed_ok(s))
    return set_error(AS_ERR_SHAPE, "bad vocab_embed shape N=%d I=%d V=%d pad_id=%d scale=%g", s->N, s->I, s->V, s->pad_id, (double)s->scale);
  if (s->dtype == AS_BF16 && s->I % 8 != 0) return set_error(AS_ERR_ALIGN, "AS_BF16 requires I %% 8 == 0 (I=%d)", s->I);
  return AS_OK;
}
bool al16e(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
as_status hip_status(hipError_t e, const char* what) {
  return e == hipSuccess ? AS_OK : set_error(AS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// threads for a row of `vecs` vectors, at most a block's
int row_threads_log(int vecs) {
  int b = 0;
  while (b < 8 && (1 << b) < vecs) ++b;
  return b;
}

hipError_t launch_sort(const vo_embed* s, const EmbedLayout& L, const int32_t* ids, unsigned char* ws, hipStream_t st) {
  auto u32 = [&](size_t at) { return reinterpret_cast<uint32_t*>(ws + at); };
  SortDev p;
  p.ids = ids;
  p.N = s->N;
  p.V = s->V;
  p.pad_id = s->pad_id;
  p.passes = L.passes;
  p.bits = L.bits;
  p.key = u32(L.key);
  p.pos = u32(L.pos);
  p.bitmap = u32(L.bitmap);
  p.bitmap_words = L.bitmap_words;
  if (L.one) {
    const size_t n64 = ((size_t)s->N + 63) & ~(size_t)63;
    const int smem = (int)(n64 * 12 + ((size_t)kSortWaves << L.bits) * 4 + kSortWaves * 4);
    static LdsLimit limit;
    const hipError_t e = limit.raise(reinterpret_cast<const void*>(sort_one_kernel), 160 * 1024);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(sort_one_kernel, dim3(1), dim3(kSortThreads), smem, st, p);
    return hipGetLastError();
  }
  // the last pass writes key / pos
  uint32_t *ka = u32(L.key), *pa = u32(L.pos), *kb = u32(L.key2), *pb = u32(L.pos2);
  if (L.passes % 2 == 0) {
    uint32_t* t = ka; ka = kb; kb = t;
    t = pa; pa = pb; pb = t;
  }
  SortPass q;
  q.key_in = q.pos_in = nullptr;
  q.places = u32(L.places);
  q.blocks = L.blocks;
  q.per = L.per;
  for (int d = 0; d < L.passes; ++d) {
    q.key_out = ka;
    q.pos_out = pa;
    q.shift = d * L.bits;
    hipLaunchKernelGGL(sort_count_kernel, dim3(L.blocks), dim3(kSortThreads), 0, st, p, q);
    hipLaunchKernelGGL(sort_places_kernel, dim3(1), dim3(kSortThreads), 0, st, p, q);
    hipLaunchKernelGGL(sort_move_kernel, dim3(L.blocks), dim3(kSortThreads), 0, st, p, q);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    q.key_in = ka;
    q.pos_in = pa;
    uint32_t* t = ka; ka = kb; kb = t;
    t = pa; pa = pb; pb = t;
  }
  return hipSuccess;
}

template <typename TE, int VEC, int PL>
hipError_t launch_sums(SumsDev p, hipStream_t st) {
  const int tpp = row_threads_log((p.I + VEC - 1) / VEC), per_block = 256 >> tpp;
  p.piece_blocks = (p.pieces + per_block - 1) / per_block;
  // (at most 2^16 rows of 2^16 columns per block and 2^20 blocks: 2^28 rows need 256 rows each at least)
  p.zero_rows = 16 * per_block;
  while ((p.V + p.zero_rows - 1) / p.zero_rows > 1 << 20) p.zero_rows *= 2;
  const int zero_blocks = p.accumulate ? 0 : (p.V + p.zero_rows - 1) / p.zero_rows;
  hipLaunchKernelGGL((embed_sums_kernel<TE, VEC, PL>), dim3(p.piece_blocks + zero_blocks), dim3(256), 0, st, p, tpp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.pieces < 2) return e;
  constexpr int CV = VEC == 1 ? 1 : 4;
  hipLaunchKernelGGL((embed_edges_kernel<TE, VEC, PL>), dim3(p.pieces, (p.I + 64 * CV - 1) / (64 * CV)), dim3(1024), 0, st, p);
  return hipGetLastError();
}
template <typename TE, int VEC> hipError_t launch_sums_any(const SumsDev& p, int L, hipStream_t st) {
  return L == 16 ? launch_sums<TE, VEC, 16>(p, st) : launch_sums<TE, VEC, 32>(p, st);
}

}  // namespace
}  // namespace asx

using namespace asx;

extern "C" size_t vocab_embed_workspace_bytes(const vo_embed* shape) {
  if (!shape || !embed_types(shape) || !embed_ok(shape) || (shape->dtype == AS_BF16 && shape->I % 8 != 0)) return 0;
  return embed_layout(shape).total;
}

extern "C" as_status vocab_embed_fwd(const vo_embed* shape, const void* table, const int32_t* ids, void* x, void* hip_stream) {
  const as_status rc = embed_check(shape);
  if (rc != AS_OK) return rc;
  if (!table || !ids || !x) return set_error(AS_ERR_NULL, "vocab_embed_fwd: a required pointer is NULL");
  if (!al16e(table) || !al16e(ids) || !al16e(x)) return set_error(AS_ERR_ALIGN, "vocab_embed_fwd: a pointer is not 16-byte aligned");
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const int N = shape->N, I = shape->I, V = shape->V;
  auto run = [&](auto* t, auto vec) {
    using TE = typename std::remove_pointer<decltype(t)>::type;
    constexpr int VEC = decltype(vec)::value;
    const int tpr = row_threads_log((I + VEC - 1) / VEC);
    const int64_t blocks = (((int64_t)N << tpr) + 255) / 256;
    hipLaunchKernelGGL((embed_fwd_kernel<TE, VEC>), dim3((unsigned)blocks), dim3(256), 0, st, reinterpret_cast<const TE*>(table),
                       ids, N, I, V, shape->pad_id, shape->scale, reinterpret_cast<TE*>(x), tpr);
    return hipGetLastError();
  };
  hipError_t e;
  if (shape->dtype == AS_BF16) e = run((uint16_t*)nullptr, std::integral_constant<int, 8>{});
  else if (I % 4 == 0) e = run((float*)nullptr, std::integral_constant<int, 4>{});
  else e = run((float*)nullptr, std::integral_constant<int, 1>{});
  return hip_status(e, "vocab_embed_fwd");
}

extern "C" as_status vocab_embed_bwd(const vo_embed* shape, const int32_t* ids, const void* dy, void* d_table, int accumulate,
                                     void* workspace, size_t workspace_bytes, void* hip_stream) {
  const as_status rc = embed_check(shape);
  if (rc != AS_OK) return rc;
  if (!ids || !dy || !d_table || !workspace) return set_error(AS_ERR_NULL, "vocab_embed_bwd: a required pointer is NULL");
  if (accumulate != 0 && accumulate != 1) return set_error(AS_ERR_SHAPE, "vocab_embed_bwd: accumulate=%d", accumulate);
  const EmbedLayout L = embed_layout(shape);
  if (workspace_bytes < L.total) return set_error(AS_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, L.total);
  if (!al16e(ids) || !al16e(dy) || !al16e(d_table) || !al16e(workspace))
    return set_error(AS_ERR_ALIGN, "vocab_embed_bwd: a pointer is not 16-byte aligned");
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  hipError_t e = launch_sort(shape, L, ids, ws, st);
  if (e != hipSuccess) return hip_status(e, "vocab_embed_bwd, sort");
  SumsDev p{};
  p.key = reinterpret_cast<const uint32_t*>(ws + L.key);
  p.pos = reinterpret_cast<const uint32_t*>(ws + L.pos);
  p.bitmap = reinterpret_cast<const uint32_t*>(ws + L.bitmap);
  p.dy = dy;
  p.d_table = d_table;
  p.edge = reinterpret_cast<float*>(ws + L.edge);
  p.N = shape->N;
  p.I = shape->I;
  p.V = shape->V;
  p.scale = shape->scale;
  p.accumulate = accumulate;
  p.pieces = L.pieces;
  if (shape->grad_dtype == AS_BF16) e = launch_sums_any<uint16_t, 8>(p, L.L, st);
  else if (shape->I % 4 == 0) e = launch_sums_any<float, 4>(p, L.L, st);
  else e = launch_sums_any<float, 1>(p, L.L, st);
  return hip_status(e, "vocab_embed_bwd");
}
