// Embedding lookup with scaling, and its gradient by sorted words (entry points and kernels).
//
// Forward: a row copy with a multiplication; bound by memory.
// Backward: d_table[v] = scale * sum of dy[n] over the positions n of word v.  Words are Zipf-like: one word has a tenth of all
// positions, most have none.  The positions are sorted by word (a stable sort, so each word's rows are added in increasing
// n, whatever the launch looks like: no float atomics), the sorted list is cut into pieces of the same length, and a group of
// threads adds up the rows of its piece, whatever words they are of.  Words that lie inside a piece are written at once; parts
// of words that reach over a piece's edge go to the workspace, and a second pass adds those up.  Rows of words that no position has
// are zeroed by further blocks of the sort's launch, or of the sums' where the radix sort takes several: d_table is written once.
#include "../../include/vocab_ops.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "common.h"
#include "lds_limit.h"
#include "row_threads.h"
#include "status.h"

namespace asx {
namespace {

typedef uint32_t eu32x4_t __attribute__((ext_vector_type(4)));

// Elements a thread moves at a time (16 bytes), as floats.  VEC < 0: rows that do not start on 16 bytes, `left` elements to their end.
// (One element at a time there and vectors, us: 66000 x 1021, 900 words, forward and backward 241 / 177, 131072 x 1023, 128000 words 663 / 472.)
// PAST: past the caches, where a call moves more than they hold (past_caches).
template <int VEC> constexpr int kWidth = VEC < 0 ? -VEC : VEC;
typedef eu32x4_t __attribute__((aligned(4))) eu32x4_on4_t;
template <typename TE, int VEC, bool PAST = false> __device__ __forceinline__ void ld_vec(const TE* p, float (&f)[kWidth<VEC>], int left) {
  if (VEC < 0 && left < kWidth<VEC>) {
#pragma unroll
    for (int i = 0; i < kWidth<VEC>; ++i) f[i] = i < left ? ld_elem<TE>(p, i) : 0.f;
    return;
  }
  using Q = typename std::conditional<(VEC < 0), eu32x4_on4_t, eu32x4_t>::type;
  const Q* from = reinterpret_cast<const Q*>(p);
  const eu32x4_t q = PAST ? __builtin_nontemporal_load(from) : *from;
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
template <typename TE, int VEC, bool PAST = false> __device__ __forceinline__ void st_vec(TE* p, const float (&f)[kWidth<VEC>], int left) {
  constexpr int W = kWidth<VEC>;
  if (VEC < 0 && left < W) {
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < left) st_elem<TE>(p, i, f[i]);
    return;
  }
  eu32x4_t q;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = sizeof(TE) == 2 ? pack_bf16(f[W / 4 * i], f[W / 4 * i + W / 4 - 1]) : __builtin_bit_cast(uint32_t, f[i]);
  using Q = typename std::conditional<(VEC < 0), eu32x4_on4_t, eu32x4_t>::type;
  if constexpr (PAST) __builtin_nontemporal_store(q, reinterpret_cast<Q*>(p));
  else *reinterpret_cast<Q*>(p) = q;
}

// the word of position n, V at padding (sorts behind all words)
__device__ __forceinline__ uint32_t word_key(const int32_t* ids, int n, int V, int pad_id) {
  const int id = ids[n];
  return id >= 0 && id < V && id != pad_id ? (uint32_t)id : (uint32_t)V;
}

// ---- forward -----------------------------------------------------------------------
// 2^tpr_log threads per row
template <typename TE, int VEC, bool PAST>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const TE* __restrict__ table, const int32_t* __restrict__ ids, int N,
                                                        int I, int V, int pad_id, float scale, TE* __restrict__ x, int tpr_log) {
  const int64_t n = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> tpr_log;
  if (n >= N) return;
  const int lane = threadIdx.x & ((1 << tpr_log) - 1), step = kWidth<VEC> << tpr_log;
  const uint32_t w = word_key(ids, (int)n, V, pad_id);
  TE* out = x + n * I;
  const TE* row = table + (int64_t)(w < (uint32_t)V ? w : 0) * I;
  for (int c = lane * kWidth<VEC>; c < I; c += step) {
    float f[kWidth<VEC>];
    if (w < (uint32_t)V) {
      ld_vec<TE, VEC>(row + c, f, I - c);
#pragma unroll
      for (int i = 0; i < kWidth<VEC>; ++i) f[i] *= scale;
    } else {
#pragma unroll
      for (int i = 0; i < kWidth<VEC>; ++i) f[i] = 0.f;
    }
    st_vec<TE, VEC, PAST>(out + c, f, I - c);
  }
}

// ---- the sort ----------------------------------------------------------------------
// Up to kRankMost positions: every position's place is the number of positions that sort ahead of it, counted by brute force over
// the whole chip: N^2 comparisons of two instructions, 3 us of arithmetic at 6400 and 14 at 16384, and one launch.  (One block that
// sorts 6400 in its LDS took 34 us.)  A wave places four positions, a lane compares every 64th vector of four keys with them.
constexpr int kRankMost = 16384, kRankBlock = 16;
struct SortDev {
  const int32_t* ids;
  int N, V, pad_id;
  uint32_t *key, *pos;   // the sorted words and positions
};
// Rows of words that no position has: a block per kZeroRows of them.
struct ZeroDev {
  void* d_table;
  int I, blocks;
};
constexpr int kZeroRows = 64;
// v0: a multiple of kZeroRows, so that these rows together start on 16 bytes whatever I is.
template <typename TE, int VEC, bool PAST>
__device__ __forceinline__ void zero_rows(TE* table, const uint8_t* has, int v0, int v1, int I, int tpp_log) {
  constexpr int W = kWidth<VEC>;
  const float zero[W] = {};
  if constexpr (VEC < 0) {   // vectors across the rows' ends where both rows are absent (inside each row: 120000 x 1001 152 us for 121)
    const uint32_t end = (uint32_t)(v1 - v0) * (uint32_t)I, width = I;
    TE* out = table + (int64_t)v0 * I;
    for (uint32_t g = threadIdx.x * W; g < end; g += 256 * W) {
      const uint32_t r = g / width;
      const bool inside = g + W <= (r + 1) * width, two = width >= W && g + W <= end;
      if (inside || two) {
        if (!has[r] && (inside || !has[r + 1])) {
          st_vec<TE, W, PAST>(out + g, zero, W);
          continue;
        }
        if (inside) continue;
      }
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (g + e < end && !has[(g + e) / width]) st_elem<TE>(out, g + e, 0.f);
    }
  } else {
    const int lane = threadIdx.x & ((1 << tpp_log) - 1), step = W << tpp_log;
    for (int v = v0 + (threadIdx.x >> tpp_log); v < v1; v += 256 >> tpp_log) {
      if (has[v - v0]) continue;
      for (int c = lane * W; c < I; c += step) st_vec<TE, VEC, PAST>(table + (int64_t)v * I + c, zero, I - c);
    }
  }
}
template <typename TE, int VEC, bool PAST> __global__ __launch_bounds__(256) void embed_rank_kernel(SortDev p, ZeroDev z, int tpp_log) {
  extern __shared__ __align__(16) uint32_t keys[];   // of all positions, to a multiple of 16
  const int N = p.N, N16 = (N + 15) & ~15, tid = threadIdx.x;
  auto key = [&](int w) { return w >= 0 && w < p.V && w != p.pad_id ? (uint32_t)w : (uint32_t)p.V; };
  auto all_ids = [&](auto use) {   // four vectors of ids together
    for (int i0 = tid * 4; i0 < N16; i0 += 4096) {
      int4 id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * 1024;
        if (i + 3 < N) {
          id[u] = *reinterpret_cast<const int4*>(p.ids + i);
        } else {
          id[u].x = i < N ? p.ids[i] : -1;
          id[u].y = i + 1 < N ? p.ids[i + 1] : -1;
          id[u].z = i + 2 < N ? p.ids[i + 2] : -1;
          id[u].w = -1;
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i0 + u * 1024 < N16) use(i0 + u * 1024, make_uint4(key(id[u].x), key(id[u].y), key(id[u].z), key(id[u].w)));
    }
  };
  const int rank_blocks = (N + kRankBlock - 1) / kRankBlock;
  if ((int)blockIdx.x >= rank_blocks) {   // they need no order: which of their rows occur, from the ids themselves
    uint8_t* has = reinterpret_cast<uint8_t*>(keys);
    const uint32_t v0 = ((int)blockIdx.x - rank_blocks) * kZeroRows;
    if (tid < kZeroRows) has[tid] = 0;
    __syncthreads();
    all_ids([&](int, uint4 k) {
      if (k.x - v0 < (uint32_t)kZeroRows) has[k.x - v0] = 1;
      if (k.y - v0 < (uint32_t)kZeroRows) has[k.y - v0] = 1;
      if (k.z - v0 < (uint32_t)kZeroRows) has[k.z - v0] = 1;
      if (k.w - v0 < (uint32_t)kZeroRows) has[k.w - v0] = 1;
    });
    __syncthreads();
    const int end = (int)v0 + kZeroRows < p.V ? (int)v0 + kZeroRows : p.V;
    zero_rows<TE, VEC, PAST>(reinterpret_cast<TE*>(z.d_table), has, (int)v0, end, z.I, tpp_log);
    return;
  }
  all_ids([&](int i, uint4 k) { *reinterpret_cast<uint4*>(keys + i) = k; });
  __syncthreads();
  const int lane = tid & 63, n0 = blockIdx.x * kRankBlock, first = n0 + (tid >> 6) * 4;   // this wave's four positions
  uint32_t mine[4], at_most[4], rank[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    mine[k] = keys[first + k];
    rank[k] = 0;
  }
  auto count = [&](uint4 q) {
#pragma unroll
    for (int k = 0; k < 4; ++k) rank[k] += (q.x < at_most[k]) + (q.y < at_most[k]) + (q.z < at_most[k]) + (q.w < at_most[k]);
  };
  // positions ahead of the block's: equal words sort ahead too
#pragma unroll
  for (int k = 0; k < 4; ++k) at_most[k] = mine[k] + 1;
#pragma unroll 4
  for (int i = lane * 4; i < n0; i += 256) count(*reinterpret_cast<const uint4*>(keys + i));
#pragma unroll
  for (int k = 0; k < 4; ++k) at_most[k] = mine[k];
#pragma unroll 4
  for (int i = n0 + kRankBlock + lane * 4; i < N16; i += 256) count(*reinterpret_cast<const uint4*>(keys + i));
  if (lane < kRankBlock) {   // the block's own
    const uint32_t q = keys[n0 + lane];
#pragma unroll
    for (int k = 0; k < 4; ++k) rank[k] += q < mine[k] + (n0 + lane < first + k ? 1u : 0u);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < 4; ++k) rank[k] += __shfl_xor(rank[k], o, 64);
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (first + k < N) {   // (what fills the last block up sorts behind everything)
        p.key[rank[k]] = mine[k];
        p.pos[rank[k]] = first + k;
      }
}

// More positions: stable radix sort of (word, position) by digits of up to 9 bits.  A wave owns a contiguous run of the keys and
// walks it 64 at a time: lanes with the same digit find each other by ballots, their rank is the number of lower such lanes, the
// wave's running count of the digit is in its own row of LDS.  Digits' places: all counts of lower digits, then those of earlier
// blocks and waves.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kDigitBits = 9, kBins = 1 << kDigitBits;

__device__ __forceinline__ uint64_t same_digit(uint32_t d, uint64_t in) {
  uint64_t m = in;
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    const uint64_t set = __ballot((d >> b) & 1u);
    m &= (d >> b) & 1u ? set : ~set;
  }
  return m;
}
__device__ __forceinline__ void lds_in_order() {   // this wave's LDS accesses before it are done before those behind it
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
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
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    const uint32_t x = waves[w];
    if (w < wave) base += x;
    sum += x;
  }
  __syncthreads();
  *total = sum;
  return base + s - v;
}

struct SortPass {
  const uint32_t *key_in, *pos_in;   // null: the first pass, from the ids
  uint32_t *key_out, *pos_out;
  uint32_t* places;                  // [digit][block]
  int blocks, per, shift;            // per: keys of a wave, a multiple of 64
};
__device__ __forceinline__ uint32_t pass_key(const SortDev& p, const SortPass& s, int i) {
  return s.key_in ? s.key_in[i] : word_key(p.ids, i, p.V, p.pad_id);
}
// f(key, position or index, whether it is one) for the wave's keys, 64 at a time, four loads ahead
template <typename F>
__device__ __forceinline__ void wave_keys(const SortDev& p, const SortPass& s, int beg, int end, F f) {
  const int lane = threadIdx.x & 63;
  for (int i0 = beg; i0 < end; i0 += 256) {
    uint32_t k[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + 64 * u + lane;
      k[u] = i < end ? pass_key(p, s, i) : 0;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + 64 * u < end) f(k[u], i0 + 64 * u + lane, i0 + 64 * u + lane < end);
  }
}
// the wave's counts of its digits
__device__ __forceinline__ void count_digits(const SortDev& p, const SortPass& s, int beg, int end, uint32_t* row) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 0; d < kBins; d += 64) row[d + lane] = 0;
  lds_in_order();
  wave_keys(p, s, beg, end, [&](uint32_t key, int, bool in) {
    const uint32_t d = (key >> s.shift) & (kBins - 1);
    const uint64_t m = same_digit(d, __ballot(in));
    if (in && (m & ((1ull << lane) - 1)) == 0) row[d] += __popcll(m);
    lds_in_order();
  });
}
__device__ __forceinline__ void wave_range(const SortDev& p, const SortPass& s, int& beg, int& end) {
  const int64_t b0 = ((int64_t)blockIdx.x * kSortWaves + (threadIdx.x >> 6)) * s.per;
  beg = b0 < p.N ? (int)b0 : p.N;
  end = b0 + s.per < p.N ? (int)(b0 + s.per) : p.N;
}
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortDev p, SortPass s) {
  __shared__ uint32_t count[kSortWaves * kBins];
  int beg, end;
  wave_range(p, s, beg, end);
  count_digits(p, s, beg, end, count + (threadIdx.x >> 6) * kBins);
  __syncthreads();
  for (int d = threadIdx.x; d < kBins; d += kSortThreads) {
    uint32_t sum = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) sum += count[w * kBins + d];
    s.places[(int64_t)d * s.blocks + blockIdx.x] = sum;
  }
}
__global__ __launch_bounds__(kSortThreads) void sort_places_kernel(SortPass s) {
  __shared__ uint32_t waves[kSortWaves];
  const int total = s.blocks * kBins;   // a multiple of 4, 2^18 at most
  uint32_t carry = 0;
  for (int i0 = 0; i0 < total; i0 += kSortThreads * 16) {   // sixteen per thread
    uint4 v[4];
    uint32_t sum = 0, all;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + threadIdx.x * 16 + u * 4;
      v[u] = i < total ? *reinterpret_cast<const uint4*>(s.places + i) : make_uint4(0, 0, 0, 0);
      sum += v[u].x + v[u].y + v[u].z + v[u].w;
    }
    uint32_t at = carry + block_prefix(sum, waves, &all);
    carry += all;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + threadIdx.x * 16 + u * 4;
      uint4 o;
      o.x = at;
      o.y = o.x + v[u].x;
      o.z = o.y + v[u].y;
      o.w = o.z + v[u].z;
      at = o.w + v[u].w;
      if (i < total) *reinterpret_cast<uint4*>(s.places + i) = o;
    }
  }
}
__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(SortDev p, SortPass s) {
  __shared__ uint32_t count[kSortWaves * kBins];
  const int lane = threadIdx.x & 63;
  uint32_t* row = count + (threadIdx.x >> 6) * kBins;
  int beg, end;
  wave_range(p, s, beg, end);
  count_digits(p, s, beg, end, row);
  __syncthreads();
  for (int d = threadIdx.x; d < kBins; d += kSortThreads) {   // counts -> the waves' first places
    uint32_t at = s.places[(int64_t)d * s.blocks + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = count[w * kBins + d];
      count[w * kBins + d] = at;
      at += c;
    }
  }
  __syncthreads();
  wave_keys(p, s, beg, end, [&](uint32_t key, int i, bool in) {
    const uint32_t d = (key >> s.shift) & (kBins - 1);
    const uint64_t m = same_digit(d, __ballot(in));
    const int rank = __popcll(m & ((1ull << lane) - 1));
    const uint32_t at = row[d] + rank;
    lds_in_order();
    if (in) {
      s.key_out[at] = key;
      s.pos_out[at] = s.key_in ? s.pos_in[i] : (uint32_t)i;
      if (rank == 0) row[d] += __popcll(m);
    }
    lds_in_order();
  });
}

// ---- the sums ----------------------------------------------------------------------
struct SumsDev {
  const uint32_t *key, *pos;
  const void* dy;
  void* d_table;
  float* edge;       // [piece][2][I]: the part of the word a piece begins within; of the word it ends within
  int N, I, V;
  float scale;
  int accumulate;
  int zero_blocks, pieces;   // zero_blocks: behind the radix sort alone
};
// first sorted place whose word is >= v, by a wave: 64 probes at a time
__device__ __forceinline__ int lower_bound_wave(const uint32_t* key, int N, uint32_t v) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = N;
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const int below = __popcll(__ballot(at < hi && key[at < hi ? at : lo] < v));
    if (below == 0) return lo;
    const int next = lo + below * step;
    lo += (below - 1) * step + 1;
    hi = next < hi ? next : hi;
  }
  return lo;
}

// 2^tpp_log (16 at least) threads per piece of L sorted positions, RU rows of it in flight: all of a short piece, whose launch is a
// few latencies long; four where the blocks of a compute unit have enough on its way together (131072 x 1024, 16 / 4: 276 / 247 us).
template <typename TE, int VEC, int L, int RU, bool PAST>
__global__ __launch_bounds__(256) void embed_sums_kernel(SumsDev p, int tpp_log) {
  __shared__ uint32_t list[2][16 * L + 1];   // the block's part of the sorted list: words, with the one ahead, and positions
  const int I = p.I, lane = threadIdx.x & ((1 << tpp_log) - 1), step = kWidth<VEC> << tpp_log;
  TE* table = reinterpret_cast<TE*>(p.d_table);
  if ((int)blockIdx.x < p.zero_blocks) {   // rows of words that no position has
    __shared__ uint8_t has[kZeroRows];
    __shared__ int range[2];
    const int v0 = (int)blockIdx.x * kZeroRows, v1 = v0 + kZeroRows < p.V ? v0 + kZeroRows : p.V, wave = threadIdx.x >> 6;
    if (wave < 2) {
      const int at = lower_bound_wave(p.key, p.N, (uint32_t)(wave == 0 ? v0 : v1));
      if ((threadIdx.x & 63) == 0) range[wave] = at;
    }
    __syncthreads();
    if (threadIdx.x < kZeroRows) {
      const uint32_t v = v0 + threadIdx.x;
      int lo = range[0], hi = range[1];
      const int end = hi;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (p.key[mid] < v) lo = mid + 1;
        else hi = mid;
      }
      has[threadIdx.x] = lo < end && p.key[lo] == v;
    }
    __syncthreads();
    zero_rows<TE, VEC, PAST>(table, has, v0, v1, I, tpp_log);
    return;
  }
  const int per_block = 256 >> tpp_log, piece0 = ((int)blockIdx.x - p.zero_blocks) * per_block, piece = piece0 + ((int)threadIdx.x >> tpp_log);
  for (int i = threadIdx.x; i < per_block * L; i += 256) {
    const int at = piece0 * L + i;
    list[0][i + 1] = at < p.N ? p.key[at] : (uint32_t)p.V;
    list[1][i] = at < p.N ? p.pos[at] : 0;
  }
  if (threadIdx.x == 0) {
    list[0][0] = piece0 > 0 ? p.key[piece0 * L - 1] : (uint32_t)p.V;
    list[1][per_block * L] = (piece0 + per_block) * L < p.N ? p.key[(piece0 + per_block) * L] : (uint32_t)p.V;   // the word behind
  }
  __syncthreads();
  if (piece >= p.pieces) return;
  const uint32_t *key = list[0] + 1 + (piece - piece0) * L, *pos = list[1] + (piece - piece0) * L;
  const uint32_t first = key[0];
  if (first >= (uint32_t)p.V) return;   // padding from here on
  const bool begins = key[-1] != first;
  const uint32_t after = piece - piece0 + 1 < per_block ? key[L] : list[1][per_block * L];
  const TE* dy = reinterpret_cast<const TE*>(p.dy);
  for (int c = lane * kWidth<VEC>; c < I; c += step) {
    float acc[kWidth<VEC>];
#pragma unroll
    for (int e = 0; e < kWidth<VEC>; ++e) acc[e] = 0.f;
    uint32_t cur = first;
    bool whole = begins;   // the run that is being added up began in this piece
    auto flush = [&](bool ends) {
      if (whole && ends) {
        float f[kWidth<VEC>];
#pragma unroll
        for (int e = 0; e < kWidth<VEC>; ++e) f[e] = acc[e] * p.scale;
        TE* out = table + (int64_t)cur * I + c;
        if (p.accumulate) {
          float old[kWidth<VEC>];
          ld_vec<TE, VEC>(out, old, I - c);
#pragma unroll
          for (int e = 0; e < kWidth<VEC>; ++e) f[e] += old[e];
        }
        st_vec<TE, VEC, PAST>(out, f, I - c);
      } else {
        float* out = p.edge + ((int64_t)piece * 2 + (whole ? 1 : 0)) * I + c;
#pragma unroll
        for (int e = 0; e < kWidth<VEC>; ++e)
          if (VEC > 0 || c + e < I) out[e] = acc[e];
      }
    };
#pragma unroll 1
    for (int u0 = 0; u0 < L; u0 += RU) {
      float x[RU][kWidth<VEC>];
      uint32_t k[RU];
#pragma unroll
      for (int u = 0; u < RU; ++u) {
        k[u] = key[u0 + u];
        if (k[u] < (uint32_t)p.V) {
          ld_vec<TE, VEC, PAST>(dy + (int64_t)pos[u0 + u] * I + c, x[u], I - c);
        } else {
#pragma unroll
          for (int e = 0; e < kWidth<VEC>; ++e) x[u][e] = 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < RU; ++u) {   // (past the list's end: padding)
        if (k[u] != cur) {
          if (cur < (uint32_t)p.V) flush(true);
          whole = true;
          cur = k[u];
#pragma unroll
          for (int e = 0; e < kWidth<VEC>; ++e) acc[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < kWidth<VEC>; ++e) acc[e] += x[u][e];
      }
    }
    if (cur < (uint32_t)p.V) flush(after != cur);
  }
}

// Words that reach over a piece's edge: the block of the piece such a word begins in adds the parts of the pieces behind it up,
// 64 threads' columns x 4 phases of every fourth piece, eight of them in flight, the phases in order.
template <typename TE, int VEC, int L>
__global__ __launch_bounds__(256) void embed_edges_kernel(SumsDev p) {
  constexpr int CV = 4, PH = 4, U = 8;
  __shared__ float red[PH][64 * CV];
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
    const float* edge = p.edge + c;
    if (phase == 0) {
#pragma unroll
      for (int e = 0; e < CV; ++e) acc[e] = VEC > 0 || c + e < I ? edge[((int64_t)piece * 2 + 1) * I + e] : 0.f;
    }
#pragma unroll 1
    for (int q0 = piece + 1 + phase; q0 < p.pieces; q0 += PH * U) {
      bool in[U];
#pragma unroll
      for (int u = 0; u < U; ++u) in[u] = q0 + PH * u < p.pieces && p.key[(q0 + PH * u) * L] == word;
      if (!in[0]) break;
      float x[U][CV];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < CV; ++e) x[u][e] = in[u] && (VEC > 0 || c + e < I) ? edge[(int64_t)(q0 + PH * u) * 2 * I + e] : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < CV; ++e) acc[e] += x[u][e];
    }
  }
#pragma unroll
  for (int e = 0; e < CV; ++e) red[phase][col * CV + e] = acc[e];
  __syncthreads();
  if (phase != 0 || c >= I) return;
#pragma unroll
  for (int q = 1; q < PH; ++q)
#pragma unroll
    for (int e = 0; e < CV; ++e) acc[e] += red[q][col * CV + e];
  TE* out = reinterpret_cast<TE*>(p.d_table) + (int64_t)word * I + c;
#pragma unroll
  for (int e = 0; e < CV; ++e) {
    if (VEC < 0 && c + e >= I) continue;
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

// Up to here pieces of 16 positions, whose launch is over in fewer latencies; behind it of 64, which are fewer edges.  us, 16 / 64: 22548 x 141 65
// / 82, 20566 x 264 bf16 64 / 79, 40000 x 512 126 / 113, 60713 x 92 84 / 75, 84157 x 648 bf16 210 / 147.
constexpr int kShortMost = 32768;

struct EmbedLayout {
  int L, pieces, passes, blocks, per;
  bool rank;
  size_t key, pos, key2, pos2, places, edge, total;
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
  L.rank = N <= kRankMost;
  L.passes = (log2_up((int64_t)s->V + 1) + kDigitBits - 1) / kDigitBits;   // words and the key of padding
  L.blocks = (N + 4095) / 4096;
  if (L.blocks > 512) L.blocks = 512;
  L.per = ((N + L.blocks - 1) / L.blocks + kSortWaves - 1) / kSortWaves;
  L.per = (L.per + 63) & ~63;
  L.L = N <= kShortMost ? 16 : 64;
  L.pieces = (N + L.L - 1) / L.L;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += upe(bytes);
    return o;
  };
  L.key = take((size_t)N * 4);
  L.pos = take((size_t)N * 4);
  L.key2 = L.pos2 = L.places = 0;
  if (!L.rank) {
    L.key2 = take((size_t)N * 4);
    L.pos2 = take((size_t)N * 4);
    L.places = take((size_t)L.blocks * kBins * 4);
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

// Streams of rows x I elements and one of `others` x I, larger than the 256 MB memory-side cache together.  131072 x 1024, 128000 words,
// fp32, forward and backward: 474 us through the caches, 442 with stores and 431 with loads past them too; below, what reads the
// result next finds it there (6400 x 512 30.3 and 33.0, 1237 x 1000 29.6 and 37.7).
bool past_caches(int64_t rows, int64_t I, int64_t e, int64_t others) { return (rows + others) * I * e > (int64_t)256 << 20; }

hipError_t launch_sort(const SortDev& p, const EmbedLayout& L, unsigned char* ws, hipStream_t st) {
  auto u32 = [&](size_t at) { return reinterpret_cast<uint32_t*>(ws + at); };
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
    q.shift = d * kDigitBits;
    hipLaunchKernelGGL(sort_count_kernel, dim3(L.blocks), dim3(kSortThreads), 0, st, p, q);
    hipLaunchKernelGGL(sort_places_kernel, dim3(1), dim3(kSortThreads), 0, st, q);
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

template <typename TE, int VEC, int PL, int RU, bool PAST>
hipError_t launch_sums(const SumsDev& p, int tpp, hipStream_t st) {
  if (tpp < 4) tpp = 4;
  const int per_block = 256 >> tpp, piece_blocks = (p.pieces + per_block - 1) / per_block;
  hipLaunchKernelGGL((embed_sums_kernel<TE, VEC, PL, RU, PAST>), dim3(p.zero_blocks + piece_blocks), dim3(256), 0, st, p, tpp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.pieces < 2) return e;
  constexpr int CV = 4;   // columns of a thread there
  hipLaunchKernelGGL((embed_edges_kernel<TE, VEC, PL>), dim3(p.pieces, (p.I + 64 * CV - 1) / (64 * CV)), dim3(256), 0, st, p);
  return hipGetLastError();
}
template <typename TE, int VEC, bool PAST>
hipError_t launch_embed_bwd(const SortDev& q, SumsDev p, const EmbedLayout& L, unsigned char* ws, hipStream_t st) {
  const int tpp = row_threads_log(p.pieces, (p.I + kWidth<VEC> - 1) / kWidth<VEC>), zero_blocks = p.accumulate ? 0 : (p.V + kZeroRows - 1) / kZeroRows;
  hipError_t e;
  if (!L.rank) {
    e = launch_sort(q, L, ws, st);
    p.zero_blocks = zero_blocks;
  } else {
    auto kfn = embed_rank_kernel<TE, VEC, PAST>;
    static LdsLimit limit;
    e = limit.raise(reinterpret_cast<const void*>(kfn), kRankMost * 4);
    if (e != hipSuccess) return e;
    const int blocks = (q.N + kRankBlock - 1) / kRankBlock;
    const size_t smem = (size_t)(blocks * kRankBlock < kZeroRows ? kZeroRows : blocks * kRankBlock) * 4;
    hipLaunchKernelGGL(kfn, dim3(blocks + zero_blocks), dim3(256), smem, st, q, ZeroDev{p.d_table, p.I, zero_blocks}, tpp);
    e = hipGetLastError();
    p.zero_blocks = 0;
  }
  if (e != hipSuccess) return e;
  return L.L == 16 ? launch_sums<TE, VEC, 16, 16, PAST>(p, tpp, st) : launch_sums<TE, VEC, 64, 4, PAST>(p, tpp, st);
}
template <typename TE, int VEC>
hipError_t launch_embed_bwd_any(const SortDev& q, const SumsDev& p, const EmbedLayout& L, unsigned char* ws, hipStream_t st) {
  return past_caches(q.N, p.I, sizeof(TE), p.accumulate ? 0 : p.V) ? launch_embed_bwd<TE, VEC, true>(q, p, L, ws, st)
                                                                 : launch_embed_bwd<TE, VEC, false>(q, p, L, ws, st);
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
    const int tpr = row_threads_log(N, (I + kWidth<VEC> - 1) / kWidth<VEC>);
    const int64_t blocks = (((int64_t)N << tpr) + 255) / 256;
    auto kfn = past_caches(N, I, sizeof(TE), 0) ? embed_fwd_kernel<TE, VEC, true> : embed_fwd_kernel<TE, VEC, false>;
    hipLaunchKernelGGL(kfn, dim3((unsigned)blocks), dim3(256), 0, st, reinterpret_cast<const TE*>(table), ids, N, I, V,
                       shape->pad_id, shape->scale, reinterpret_cast<TE*>(x), tpr);
    return hipGetLastError();
  };
  hipError_t e;
  if (shape->dtype == AS_BF16) e = run((uint16_t*)nullptr, std::integral_constant<int, 8>{});
  else if (I % 4 == 0) e = run((float*)nullptr, std::integral_constant<int, 4>{});
  else e = run((float*)nullptr, std::integral_constant<int, -4>{});
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
  SortDev q;
  q.ids = ids;
  q.N = shape->N;
  q.V = shape->V;
  q.pad_id = shape->pad_id;
  q.key = reinterpret_cast<uint32_t*>(ws + L.key);
  q.pos = reinterpret_cast<uint32_t*>(ws + L.pos);
  SumsDev p{};
  p.key = q.key;
  p.pos = q.pos;
  p.dy = dy;
  p.d_table = d_table;
  p.edge = reinterpret_cast<float*>(ws + L.edge);
  p.N = shape->N;
  p.I = shape->I;
  p.V = shape->V;
  p.scale = shape->scale;
  p.accumulate = accumulate;
  p.pieces = L.pieces;
  hipError_t e;
  if (shape->grad_dtype == AS_BF16) e = launch_embed_bwd_any<uint16_t, 8>(q, p, L, ws, st);
  else if (shape->I % 4 == 0) e = launch_embed_bwd_any<float, 4>(q, p, L, ws, st);
  else e = launch_embed_bwd_any<float, -4>(q, p, L, ws, st);
  return hip_status(e, "vocab_embed_bwd");
}
