// Verification of drafted words against the target's probabilities (speculative sampling): entry points and kernels.
//
// A word is told from its neighbour by where a random number falls among sums over the vocabulary, so that probabilities are computed
// in 64 bits: with 128000 borders, each off by 1e-8 as in fp32, one draw in a thousand would go to another word.  fp64 instructions run at
// nearly fp32's rate here (additions 34e12 of a lane a second, with a multiplication 32e12; in fp32 36e12 and 34e12).
// Two launches.  The first one reads all rows once, a chunk of a row per block: its maximum and the sum of exp relative to it.  In
// the second every block of a sequence joins those, finds how many words are accepted, and, where one was refused, adds up the weights
// max(p - q, 0) of its chunk; the sequence's last block to arrive finds the chunk in which u times the sum lies, and in it the word.
#include "../../include/vocab_ops.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "common.h"
#include "status.h"

namespace asx {
namespace {

typedef uint32_t vu32x4_t __attribute__((ext_vector_type(4)));

constexpr int kVThreads = 256, kVerifyMaxT = 64;
// Logits of a thread: a block's chunk of a row is 256 times that.  Fewer where the blocks would not fill the chip: see verify_layout.
constexpr int kManyPer = 32, kFewPer = 8, kMostChunks = 128;   // (two to a lane of the wave that scans their sums)
constexpr int kMostTries = 100000;                                // of reading a sum

struct VerifyPart {
  double sum;    // of 2^((l - m) c)
  float m;
  int32_t bad;   // a NaN or +inf among them
};
struct VerifyDev {
  const void *target, *draft;
  int64_t ld_target, ld_draft;
  const int32_t* drafted;
  const float *u_accept, *u_next;
  int32_t *n_accepted, *words;
  VerifyPart* part;    // [B][2T+1][chunks]: T+1 rows of the target, T of the draft
  double* sums;        // [B][chunks]: of max(p - q, 0); below 0: not there yet
  uint32_t* ticket;    // [B]
  int32_t B, T, V, chunks;
  double c;            // log2(e) / tau
};

// 2^y by the exponential's series of y's fractional part, |f ln 2| <= 0.347: the first term left out is 6e-15 of the result
__device__ __forceinline__ double exp2_64(double y) {
  y = fmax(y, -1100.0);   // (0; -inf too)
  const double n = rint(y), f = y - n;
  double p = 4.4455382718708115e-10;                     // ln(2)^k / k!, k = 11 .. 0
  p = fma(p, f, 7.0549116208011233e-09);
  p = fma(p, f, 1.0178086009239700e-07);
  p = fma(p, f, 1.3215486790144309e-06);
  p = fma(p, f, 1.5252733804059841e-05);
  p = fma(p, f, 1.5403530393381608e-04);
  p = fma(p, f, 1.3333558146428443e-03);
  p = fma(p, f, 9.6181291076284772e-03);
  p = fma(p, f, 5.5504108664821580e-02);
  p = fma(p, f, 2.4022650695910072e-01);
  p = fma(p, f, 6.9314718055994531e-01);
  p = fma(p, f, 1.0);
  return ldexp(p, (int)n);
}

// The same with the powers 2^(k / 256), k = 0 .. 255, in a table: what is left of y is 2^-9 at most, and the first term left out 1.4e-13 of the
// result.  Eight fp64 instructions, four of 32 bits and a read of LDS in place of 16 fp64 ones.
constexpr int kPowers = 256;
__device__ __forceinline__ void make_powers(double* powers) { powers[threadIdx.x] = exp2_64((double)threadIdx.x / kPowers); }
__device__ __forceinline__ double exp2_by_powers(double y, const double* powers) {
  constexpr double kMagic = 0x1.8p44;    // its last place is 2^-8
  // y >= -1100.02: of negative numbers the larger words are the lower ones (2^y is 0 from there on; -inf too)
  uint64_t bits = __builtin_bit_cast(uint64_t, y);
  const uint32_t high = (uint32_t)(bits >> 32);
  bits = (bits & 0xffffffffu) | (uint64_t)(high < 0xc0913000u ? high : 0xc0913000u) << 32;
  y = __builtin_bit_cast(double, bits);
  const double z = y + kMagic, r = y - (z - kMagic);
  const int k = (int)(uint32_t)__builtin_bit_cast(uint64_t, z);
  const double t = powers[k & (kPowers - 1)];
  double q = fma(5.5504108664821580e-02, r, 2.4022650695910072e-01);
  q = fma(q, r, 6.9314718055994531e-01) * r;
  return ldexp(fma(t, q, t), k >> 8);
}

// Of 2 to the power of this: the difference first, which is 0 at l = m.  Were c m taken off c l, its rounding would be in the exponent, 1e22 of
// them at the lowest float, and such are what excluded words are given.
__device__ __forceinline__ double exponent(float l, float m, double c) { return ((double)l - (double)m) * c; }

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// l[0 .. 16 / sizeof(TE)) = the vector at v0 of a row, -inf behind its end (rows may end with the memory: no element behind V is read)
template <typename TE> __device__ __forceinline__ void ld_logits(const TE* row, int v0, int V, float* l) {
  constexpr int W = 16 / sizeof(TE);
  if (v0 + W <= V) {
    const vu32x4_t q = *reinterpret_cast<const vu32x4_t*>(row + v0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = q[i];
      if constexpr (sizeof(TE) == 2) {
        l[2 * i] = lo_bf16(w);
        l[2 * i + 1] = hi_bf16(w);
      } else {
        l[i] = __builtin_bit_cast(float, w);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) l[i] = v0 + i < V ? ld_elem<TE>(row, v0 + i) : -INFINITY;
  }
}

__device__ __forceinline__ bool is_word(int32_t x, int V) { return x >= 0 && x < V; }

// ---- statistics of the rows --------------------------------------------------------
template <typename TE, int PER> __global__ __launch_bounds__(kVThreads) void verify_stats_kernel(VerifyDev a) {
  constexpr int W = 16 / sizeof(TE);
  __shared__ float s_m[4];
  __shared__ double s_sum[4], s_powers[kPowers];
  const int rows = 2 * a.T + 1, b = blockIdx.y / rows, j = blockIdx.y - b * rows;
  const int tid = threadIdx.x, wave = tid >> 6;
  if (j == 0 && tid == 0) {
    a.sums[(int64_t)b * a.chunks + blockIdx.x] = -1.0;
    if (blockIdx.x == 0) a.ticket[b] = 0;
  }
  // the target's row t is looked at behind t words, the draft's with its word
  const int t = j <= a.T ? j : j - a.T - 1, ahead = j <= a.T ? t : t + 1;
  for (int i = 0; i < ahead; ++i)
    if (!is_word(a.drafted[(int64_t)b * a.T + i], a.V)) return;
  const TE* row = j <= a.T ? reinterpret_cast<const TE*>(a.target) + ((int64_t)b * (a.T + 1) + t) * a.ld_target
                           : reinterpret_cast<const TE*>(a.draft) + ((int64_t)b * a.T + t) * a.ld_draft;
  float l[PER];
#pragma unroll
  for (int i = 0; i < PER / W; ++i) {
    const int v0 = blockIdx.x * kVThreads * PER + (i * kVThreads + tid) * W;
    ld_logits<TE>(row, v0 < a.V ? v0 : a.V, a.V, l + i * W);
  }
  make_powers(s_powers);                   // (while the logits are on their way)
  float m = -INFINITY;
  int bad = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    m = fmaxf(m, l[i]);
    bad |= !(l[i] < INFINITY);
  }
  m = wave_max(m);
  bad = __syncthreads_or(bad);
  if ((tid & 63) == 0) s_m[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  double sum = 0;
  if (m > -INFINITY && !bad) {
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += exp2_by_powers(exponent(l[i], m, a.c), s_powers);
  }
  sum = wave_sum64(sum);
  if ((tid & 63) == 0) s_sum[wave] = sum;
  __syncthreads();
  if (tid == 0) a.part[(int64_t)blockIdx.y * a.chunks + blockIdx.x] = {(s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]), m, bad};
}

// The same of many bf16 logits.  Of those there are few different ones: 24 exponents of 128 and two signs are a table of 48 KB, which
// takes the place of an exponential each by a read of LDS; it is made once by blocks that stay for all chunks.  Sums are relative to
// 2^0 instead of the chunk's maximum.  A chunk with other logits (64 and more in magnitude, 2^-18 and less, infinities, NaN) goes the general
// way.  us, 1152 rows of 128000 (295 MB): the general way 120, this 84, of which the vector units and LDS (a quarter of its time conflicts of
// banks) are busy 55 each.
constexpr int kTabThreads = 512, kTabPer = 16, kTabBlocks = 768;
constexpr uint32_t kTabFirst = (127 - 18) << 7, kTabCount = 24 << 7;   // the lowest magnitude's bits, how many
constexpr double kTabMost = 1000.0;                                    // 64 c: powers and sums of 2^20 of them are in fp64's range
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
__global__ __launch_bounds__(kTabThreads) void verify_stats_table_kernel(VerifyDev a) {
  static_assert(kTabThreads * kTabPer == kVThreads * kManyPer && 16 * (kTabCount + 1) < 1 << 16, "the same chunks; places in 16 bits");
  constexpr int WAVES = kTabThreads / 64;
  __shared__ double s_table[2 * (kTabCount + 1)];   // positive and negative ones in turns; zeros for what is not in it
  __shared__ double s_powers[kPowers], s_sum[2][WAVES];
  __shared__ int s_odd[2][WAVES];
  __shared__ float s_m[WAVES];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, rows = 2 * a.T + 1;
  if (tid < kPowers) make_powers(s_powers);
  for (int i = tid; i < 2 * ((int)kTabCount + 1); i += kTabThreads) {
    const double l = bf16_bits_to_f32((uint32_t)(i >> 1) + kTabFirst | (uint32_t)(i & 1) << 15);
    s_table[i] = i >> 1 < (int)kTabCount ? exp2_64(l * a.c) : 0.0;
  }
  // (a block for each sequence: by all threads of all blocks, the compiler's code for the loop below took 101 us instead of 91)
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    if (tid < a.chunks) a.sums[(int64_t)b * a.chunks + tid] = -1.0;
    if (tid == 0) a.ticket[b] = 0;
  }
  __syncthreads();
  // An item is a chunk of a row.  While one is added up, the next one's logits are on their way, and the drafted words that say whether
  // the one behind it is looked at at all.
  struct Item {
    int b, j, chunk;
  };
  auto item_at = [&](int n) {
    Item i;
    const int row = n / a.chunks;
    i.chunk = n - row * a.chunks;
    i.b = row / rows;
    i.j = row - i.b * rows;
    return i;
  };
  const Item step = item_at(gridDim.x);
  auto behind = [&](Item i) {              // (divisions in every step kept the scalar unit busier than the vector units)
    i.chunk += step.chunk;
    i.j += step.j;
    i.b += step.b;
    if (i.chunk >= a.chunks) {
      i.chunk -= a.chunks;
      ++i.j;
    }
    if (i.j >= rows) {
      i.j -= rows;
      ++i.b;
    }
    return i;
  };
  auto ask = [&](const Item& i) {          // drafted words of the item's sequence, a lane each
    return lane < a.T && i.b < a.B ? a.drafted[(int64_t)i.b * a.T + lane] : -1;
  };
  vu32x4_t next[2];
  bool next_there[2];
  auto load = [&](const Item& i, int32_t word) {
    next_there[0] = next_there[1] = false;
    if (i.b >= a.B) return;
    const int t = i.j <= a.T ? i.j : i.j - a.T - 1, ahead = i.j <= a.T ? t : t + 1;
    const uint64_t none = ~__ballot(is_word(word, a.V));
    if (none && __builtin_ctzll(none) < ahead) return;
    const uint16_t* from = i.j <= a.T ? reinterpret_cast<const uint16_t*>(a.target) + ((int64_t)i.b * (a.T + 1) + t) * a.ld_target
                                      : reinterpret_cast<const uint16_t*>(a.draft) + ((int64_t)i.b * a.T + t) * a.ld_draft;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int v = i.chunk * (kTabThreads * kTabPer) + (h * kTabThreads + tid) * 8;
      next_there[h] = v < a.V;
      if (v + 8 <= a.V) {
        next[h] = *reinterpret_cast<const vu32x4_t*>(from + v);
      } else if (v < a.V) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t lo = v + 2 * k < a.V ? from[v + 2 * k] : 0xff80u, hi = v + 2 * k + 1 < a.V ? from[v + 2 * k + 1] : 0xff80u;
          next[h][k] = lo | hi << 16;
        }
      }
    }
  };
  Item i0 = item_at(blockIdx.x), i1 = behind(i0);
  load(i0, ask(i0));
  int32_t word = ask(i1);
  int par = 0;
  for (; i0.b < a.B; i0 = i1, i1 = behind(i1), par ^= 1) {
    const int64_t at = ((int64_t)i0.b * rows + i0.j) * a.chunks + i0.chunk;
    vu32x4_t x[2];
    bool there[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[h] = next[h];
      there[h] = next_there[h];
    }
    load(i1, word);
    word = ask(behind(i1));
    // two logits at a time: places in the table, in bytes
    double sum = 0, sum2 = 0;
    u16x2_t most = {0, 0};
    constexpr u16x2_t kFirst = {kTabFirst, kTabFirst}, kCount = {kTabCount, kTabCount};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!there[h]) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = x[h][i];
        const u16x2_t u = __builtin_elementwise_min((u16x2_t)(__builtin_bit_cast(u16x2_t, w & 0x7fff7fffu) - kFirst), kCount);   // (below: wraps)
        most = __builtin_elementwise_max(most, u);
        const uint32_t at = __builtin_bit_cast(uint32_t, (u16x2_t)(u * (uint16_t)16 + __builtin_bit_cast(u16x2_t, w >> 12 & 0x00080008u)));
        sum += *reinterpret_cast<const double*>(reinterpret_cast<const unsigned char*>(s_table) + (at & 0xffffu));
        sum2 += *reinterpret_cast<const double*>(reinterpret_cast<const unsigned char*>(s_table) + (at >> 16));
      }
    }
    const bool odd = __any(most[0] == kTabCount || most[1] == kTabCount);
    sum = wave_sum64(sum + sum2);
    if (lane == 0) {
      s_sum[par][wave] = sum;
      s_odd[par][wave] = odd;
    }
    __syncthreads();
    int any_odd = 0;
    sum = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      any_odd |= s_odd[par][w];
      sum += s_sum[par][w];
    }
    if (!any_odd) {
      if (tid == 0) a.part[at] = {sum, 0.f, 0};
      continue;
    }
    // the general way
    float m = -INFINITY;
    int bad = 0;
    float l[kTabPer];
#pragma unroll
    for (int k = 0; k < kTabPer; ++k) {
      const uint32_t w = x[k / 8][k % 8 / 2];
      l[k] = there[k / 8] ? (k % 2 ? hi_bf16(w) : lo_bf16(w)) : -INFINITY;
      m = fmaxf(m, l[k]);
      bad |= !(l[k] < INFINITY);
    }
    m = wave_max(m);
    bad = __syncthreads_or(bad);
    if (lane == 0) s_m[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, s_m[w]);
    sum = 0;
    if (m > -INFINITY && !bad) {
#pragma unroll
      for (int k = 0; k < kTabPer; ++k) sum += exp2_by_powers(exponent(l[k], m, a.c), s_powers);
    }
    sum = wave_sum64(sum);
    __syncthreads();
    if (lane == 0) s_sum[par][wave] = sum;
    __syncthreads();
    if (tid == 0) {
      sum = 0;
      for (int w = 0; w < WAVES; ++w) sum += s_sum[par][w];
      a.part[at] = {sum, m, bad};
    }
  }
}

// ---- the words ---------------------------------------------------------------------
template <typename TE, int PER> __global__ __launch_bounds__(kVThreads, 8) void verify_words_kernel(VerifyDev a) {
  constexpr int W = 16 / sizeof(TE), CHUNK = kVThreads * PER;
  __shared__ double s_lift[2 * kVerifyMaxT + 1];     // p[v] = 2^((l[v] - top) c + lift)
  __shared__ float s_top[2 * kVerifyMaxT + 1];
  __shared__ int8_t s_bad[2 * kVerifyMaxT + 1];
  // (single values are written in one place each: no wave can be late to read what was there before)
  __shared__ int s_words, s_n, s_state, s_last, s_chunk, s_of_p, s_past[kVThreads / 64], s_some[kVThreads / 64];
  __shared__ double s_r[4], s_ahead, s_theta, s_powers[kPowers];
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, T = a.T, V = a.V;
  const int64_t first = (int64_t)b * T;
  const TE* target = reinterpret_cast<const TE*>(a.target) + (int64_t)b * (T + 1) * a.ld_target;
  const TE* draft = reinterpret_cast<const TE*>(a.draft) + first * a.ld_draft;
  // the drafted words, their logits and random numbers: a lane of the first wave each
  float lp_x = 0.f, lq_x = 0.f, u = 0.f;
  if (wave == 0) {
    const int32_t x = lane < T ? a.drafted[first + lane] : -1;
    const bool given = is_word(x, V);
    if (given) {
      lp_x = ld_elem<TE>(target + lane * a.ld_target, x);
      lq_x = ld_elem<TE>(draft + lane * a.ld_draft, x);
      u = a.u_accept[first + lane];
    }
    const uint64_t none = ~__ballot(given);
    if (lane == 0) s_words = none ? __builtin_ctzll(none) : 64;
  }
  make_powers(s_powers);
  __syncthreads();
  const int words = s_words;
  // 16 lanes join the parts of a row
  for (int i = tid >> 4; i < 2 * words + 1; i += kVThreads / 16) {
    const int j = i <= words ? i : i - words + T;   // (target rows 0 .. words, draft rows 0 .. words - 1)
    const VerifyPart* part = a.part + ((int64_t)b * (2 * T + 1) + j) * a.chunks;
    float m = -INFINITY;
    int bad = 0;
    double z = 0;                                   // relative to the lane's own maximum
    for (int k = lane & 15; k < a.chunks; k += 16) {
      const VerifyPart x = part[k];
      bad |= x.bad;
      const float up = fmaxf(m, x.m);
      if (up > -INFINITY)
        z = (m > -INFINITY ? z * exp2_by_powers(exponent(m, up, a.c), s_powers) : 0.0) +
            (x.m > -INFINITY ? x.sum * exp2_by_powers(exponent(x.m, up, a.c), s_powers) : 0.0);
      m = up;
    }
    float top = m;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      top = fmaxf(top, __shfl_xor(top, o, 64));
      bad |= __shfl_xor(bad, o, 64);
    }
    z = m > -INFINITY ? z * exp2_by_powers(exponent(m, top, a.c), s_powers) : 0.0;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) z += __shfl_xor(z, o, 64);
    if ((lane & 15) == 0) {
      s_top[j] = top;
      s_lift[j] = -log2(z);
      s_bad[j] = bad || !(top > -INFINITY);
    }
  }
  __syncthreads();
  if (wave == 0) {
    bool ok = false, bad = false;
    if (lane < words) {
      bad = s_bad[lane] || s_bad[T + 1 + lane];
      ok = !bad && (double)u * exp2_by_powers(exponent(lq_x, s_top[T + 1 + lane], a.c) + s_lift[T + 1 + lane], s_powers) <
                       exp2_by_powers(exponent(lp_x, s_top[lane], a.c) + s_lift[lane], s_powers);
    }
    const uint64_t not_ok = ~__ballot(ok), bads = __ballot(bad);
    if (lane == 0) {
      const int n = not_ok ? __builtin_ctzll(not_ok) : 64;
      s_n = n;
      s_state = (n < words && (bads >> n & 1)) || s_bad[n] ? 2 : n < words;   // 0: from p, 1: what is left of p, 2: no distribution
    }
  }
  __syncthreads();
  const int n = s_n, state = s_state;
  const bool rest = state == 1;
  if (blockIdx.x == 0) {
    if (tid == 0) a.n_accepted[b] = n;
    if (tid <= T && (tid != n || state == 2)) a.words[first + b + tid] = tid < n ? a.drafted[first + tid] : -1;
  }
  if (state == 2) return;
  const TE *p_row = target + n * a.ld_target, *q_row = draft + (rest ? n : 0) * a.ld_draft;
  const float p_top = s_top[n], q_top = s_top[rest ? T + 1 + n : n];
  const double p_lift = s_lift[n], q_lift = s_lift[rest ? T + 1 + n : n];
  // what counts of a word: all of p, or what is above q
  auto weight = [&](auto subtract, float lp, float lq) {
    const double p = exp2_by_powers(exponent(lp, p_top, a.c) + p_lift, s_powers);
    if constexpr (!decltype(subtract)::value) return p;
    else return fmax(p - exp2_by_powers(exponent(lq, q_top, a.c) + q_lift, s_powers), 0.0);
  };
  // weights of the words from v0 on, vectors step words apart
  auto weights = [&](auto subtract, int v0, int step) {
    double sum = 0;
#pragma unroll 1
    for (int i = 0; i < PER / W; ++i, v0 += step) {
      float lp[W], lq[W] = {};
      ld_logits<TE>(p_row, v0 < V ? v0 : V, V, lp);
      if constexpr (decltype(subtract)::value) ld_logits<TE>(q_row, v0 < V ? v0 : V, V, lq);
#pragma unroll
      for (int e = 0; e < W; ++e) sum += weight(subtract, lp[e], lq[e]);
    }
    return sum;
  };
  double* sums = a.sums + (int64_t)b * a.chunks;
  if (rest) {
    // this chunk's
    double r = weights(std::true_type{}, blockIdx.x * CHUNK + tid * W, kVThreads * W);
    r = wave_sum64(r);
    if (lane == 0) s_r[wave] = r;
    __syncthreads();
    if (tid == 0) {
      __hip_atomic_store(&sums[blockIdx.x], (s_r[0] + s_r[1]) + (s_r[2] + s_r[3]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // The ticket orders nothing: the last block reads the sums, and nothing else that other blocks of this launch write, until each is there.
      // (As a release it writes the L2 back, for every block: 160 -> 143 us at 128 x 4 words of 128000, 36 -> 31 at 37 x 5 of 32003.)
      s_last = __hip_atomic_fetch_add(&a.ticket[b], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.chunks - 1;
    }
    __syncthreads();
    if (!s_last) return;
  } else if (blockIdx.x != 0) {
    return;                            // p's chunks have been added up by the statistics
  }
  // One block, the sequence's last or first, finds the chunk; sums are added in the chunks' order, whichever block this is.
  if (wave == 0) {
    double x[2], run[2], all = 0;
    bool missing = false;
    auto scan = [&]() {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        run[h] = x[h];
        if (h == 1 && a.chunks <= 64) {
          run[1] = run[0];
          break;
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const double y = __shfl_up(run[h], o, 64);
          if (lane >= o) run[h] += y;
        }
        if (h == 1) run[1] += __shfl(run[0], 63, 64);
      }
      all = __shfl(run[1], 63, 64);
    };
    if (rest) {
      // Every block has counted, and stores its sum ahead of that or soon after, waiting for nobody.  Some 1e5 reads of 1 us each find one
      // missing only where another call takes the workspace meanwhile, which no caller may do: no word then, but an end.
      int tries = 0;
      do {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = h * 64 + lane;
          x[h] = k < a.chunks ? __hip_atomic_load(&sums[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
        }
      } while ((x[0] < 0 || x[1] < 0) && ++tries < kMostTries);
      missing = __any(x[0] < 0 || x[1] < 0);
      scan();
    }
    const bool of_p = !(all > 0);           // nothing is left: p
    if (of_p) {
      const VerifyPart* part = a.part + ((int64_t)b * (2 * T + 1) + n) * a.chunks;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = h * 64 + lane;
        x[h] = 0.0;
        if (k < a.chunks && part[k].m > -INFINITY) x[h] = part[k].sum * exp2_by_powers(exponent(part[k].m, p_top, a.c) + p_lift, s_powers);
      }
      scan();
    }
    const double theta = fmax((double)a.u_next[b], 0.0) * all;
    int chunk = -1, some = 0;
    double left = INFINITY;
#pragma unroll
    for (int h = 1; h >= 0; --h) {
      const double own = x[h];
      const uint64_t above = __ballot(own > 0 && run[h] > theta), there = __ballot(own > 0);   // (of weight 0: rounding alone)
      if (above) {
        const int k = __builtin_ctzll(above);
        chunk = h * 64 + k;
        left = theta - __shfl(run[h] - own, k, 64);
      }
      if (there && some == 0) some = h * 64 + 63 - __builtin_clzll(there);
    }
    if (lane == 0) {
      s_chunk = missing ? -1 : chunk < 0 ? some : chunk;   // (rounding, or u >= 1: the last one with a weight)
      s_theta = left;
      s_of_p = of_p;
    }
  }
  __syncthreads();
  if (s_chunk < 0) {
    if (tid == 0) a.words[first + b + n] = -1;
    return;
  }
  const bool subtract = !s_of_p;
  const int v1 = s_chunk * CHUNK + tid * PER;   // consecutive logits per thread: running sums go by the words' order
  const double theta = s_theta;
  const double own = subtract ? weights(std::true_type{}, v1, W) : weights(std::false_type{}, v1, W);
  double run = own;   // inclusive over the block
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double x = __shfl_up(run, o, 64);
    if (lane >= o) run += x;
  }
  if (lane == 63) s_r[wave] = run;
  __syncthreads();
  for (int i = 0; i < wave; ++i) run += s_r[i];
  // the first thread past theta, and the last one with a weight
  const uint64_t past = __ballot(own > 0 && run > theta), some = __ballot(own > 0);
  if (lane == 0) {
    s_past[wave] = past ? wave * 64 + __builtin_ctzll(past) : kVThreads;
    s_some[wave] = some ? wave * 64 + 63 - __builtin_clzll(some) : -1;
  }
  __syncthreads();
  int at = kVThreads, last = -1;
#pragma unroll
  for (int i = 0; i < kVThreads / 64; ++i) {
    at = s_past[i] < at ? s_past[i] : at;
    last = s_some[i] > last ? s_some[i] : last;
  }
  const bool none = at == kVThreads;         // (as above: the chunk's last word of a weight above 0)
  if (none) at = last > 0 ? last : 0;
  if (tid == at) s_ahead = run - own;
  __syncthreads();
  if (wave != 0) return;
  // that thread's words, a lane each
  const int v = s_chunk * CHUNK + at * PER + lane;
  double mine = 0;
  if (lane < PER && v < V) {
    const float lp = ld_elem<TE>(p_row, v), lq = subtract ? ld_elem<TE>(q_row, v) : 0.f;
    mine = subtract ? weight(std::true_type{}, lp, lq) : weight(std::false_type{}, lp, lq);
  }
  run = mine;
#pragma unroll
  for (int o = 1; o < PER; o <<= 1) {
    const double x = __shfl_up(run, o, 64);
    if (lane >= o) run += x;
  }
  const uint64_t above = __ballot(!none && mine > 0 && s_ahead + run > theta), there = __ballot(mine > 0);
  if (lane == 0) a.words[first + b + n] = s_chunk * CHUNK + at * PER + (above ? __builtin_ctzll(above) : there ? 63 - __builtin_clzll(there) : 0);
}

struct VerifyLayout {
  int per, chunks;
  size_t part, sums, ticket, total;
};
VerifyLayout verify_layout(const vo_verify* s) {
  VerifyLayout L;
  // us, the whole call, 32 / 8 logits a thread: 4 words of one sentence of 32000 28 / 18, 37 x 5 of 32003 in fp32 37 / 35; 128 x 4 of 128000 only 32.
  const int64_t few = kVThreads * kFewPer;
  L.per = (int64_t)s->B * (2 * s->T + 1) * ((s->V + few - 1) / few) <= 8192 && s->V <= few * kMostChunks ? kFewPer : kManyPer;
  L.chunks = (s->V + kVThreads * L.per - 1) / (kVThreads * L.per);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  L.part = 0;
  L.sums = up((size_t)s->B * (2 * s->T + 1) * L.chunks * sizeof(VerifyPart));
  L.ticket = L.sums + up((size_t)s->B * L.chunks * sizeof(double));
  L.total = L.ticket + up((size_t)s->B * 4);
  return L;
}
bool verify_ok(const vo_verify* s) {
  return s->B >= 1 && s->B <= (1 << 16) && s->T >= 1 && s->T <= kVerifyMaxT && s->V >= 1 && s->V <= (1 << 20) &&
         s->temperature >= 0x1p-10f && s->temperature <= 0x1p10f;
}
bool verify_types(const vo_verify* s) { return s->dtype == AS_F32 || s->dtype == AS_BF16; }
bool al16r(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename TE, int PER> hipError_t launch_verify(const VerifyDev& d, hipStream_t st) {
  // rows of a launch: the grid's second dimension takes 65535
  const int rows = 2 * d.T + 1, most = 65535 / rows;
  for (int b0 = 0; b0 < d.B; b0 += most) {
    VerifyDev p = d;
    p.B = d.B - b0 < most ? d.B - b0 : most;
    p.target = reinterpret_cast<const TE*>(d.target) + (int64_t)b0 * (d.T + 1) * d.ld_target;
    p.draft = reinterpret_cast<const TE*>(d.draft) + (int64_t)b0 * d.T * d.ld_draft;
    p.drafted += (int64_t)b0 * d.T;
    p.u_accept += (int64_t)b0 * d.T;
    p.u_next += b0;
    p.n_accepted += b0;
    p.words += (int64_t)b0 * (d.T + 1);
    p.part += (int64_t)b0 * rows * d.chunks;
    p.sums += (int64_t)b0 * d.chunks;
    p.ticket += b0;
    hipError_t e;
    if (sizeof(TE) == 2 && PER == kManyPer && d.c * 64 <= kTabMost && (int64_t)p.B * rows * d.chunks >= 4 * kTabBlocks) {
      hipLaunchKernelGGL(verify_stats_table_kernel, dim3(kTabBlocks), dim3(kTabThreads), 0, st, p);
    } else {
      hipLaunchKernelGGL((verify_stats_kernel<TE, PER>), dim3(d.chunks, p.B * rows), dim3(kVThreads), 0, st, p);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((verify_words_kernel<TE, PER>), dim3(d.chunks, p.B), dim3(kVThreads), 0, st, p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace
}  // namespace asx

using namespace asx;

extern "C" size_t vocab_verify_workspace_bytes(const vo_verify* shape) {
  if (!shape || !verify_types(shape) || !verify_ok(shape)) return 0;
  return verify_layout(shape).total;
}

extern "C" as_status vocab_verify(const vo_verify* shape, const void* target, int64_t ld_target, const void* draft, int64_t ld_draft,
                                  const int32_t* drafted, const float* u_accept, const float* u_next, int32_t* n_accepted, int32_t* words,
                                  void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!shape) return set_error(AS_ERR_NULL, "shape is NULL");
  if (!verify_types(shape)) return set_error(AS_ERR_DTYPE, "vocab_verify: dtype %d", shape->dtype);
  if (!verify_ok(shape))
    return set_error(AS_ERR_SHAPE, "bad shape B=%d T=%d V=%d temperature=%g", shape->B, shape->T, shape->V, (double)shape->temperature);
  if (!target || !draft || !drafted || !u_accept || !u_next || !n_accepted || !words || !workspace)
    return set_error(AS_ERR_NULL, "vocab_verify: a required pointer is NULL");
  const int64_t e = shape->dtype == AS_F32 ? 4 : 2;
  for (int64_t ld : {ld_target, ld_draft}) {
    if (ld < shape->V || ld >= (int64_t)1 << 40) return set_error(AS_ERR_SHAPE, "vocab_verify: rows of %d logits %lld apart", shape->V, (long long)ld);
    if (ld * e % 16 != 0) return set_error(AS_ERR_ALIGN, "vocab_verify: rows %lld elements apart do not start on 16 bytes", (long long)ld);
  }
  const VerifyLayout L = verify_layout(shape);
  if (workspace_bytes < L.total) return set_error(AS_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, L.total);
  for (const void* p : {target, draft, (const void*)drafted, (const void*)u_accept, (const void*)u_next, (const void*)n_accepted, (const void*)words,
                        (const void*)workspace})
    if (!al16r(p)) return set_error(AS_ERR_ALIGN, "vocab_verify: a pointer is not 16-byte aligned");
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  VerifyDev d;
  d.target = target;
  d.draft = draft;
  d.ld_target = ld_target;
  d.ld_draft = ld_draft;
  d.drafted = drafted;
  d.u_accept = u_accept;
  d.u_next = u_next;
  d.n_accepted = n_accepted;
  d.words = words;
  d.part = reinterpret_cast<VerifyPart*>(ws + L.part);
  d.sums = reinterpret_cast<double*>(ws + L.sums);
  d.ticket = reinterpret_cast<uint32_t*>(ws + L.ticket);
  d.B = shape->B;
  d.T = shape->T;
  d.V = shape->V;
  d.chunks = L.chunks;
  d.c = 1.4426950408889634 / (double)shape->temperature;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const bool few = L.per == kFewPer;
  const hipError_t err = e == 4 ? (few ? launch_verify<float, kFewPer>(d, st) : launch_verify<float, kManyPer>(d, st))
                                : (few ? launch_verify<uint16_t, kFewPer>(d, st) : launch_verify<uint16_t, kManyPer>(d, st));
  return err == hipSuccess ? AS_OK : set_error(AS_ERR_HIP, "vocab_verify: %s", hipGetErrorString(err));
}
