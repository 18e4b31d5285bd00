// Few rows (a decoder step): the projection's softmax statistics in one pass over W, the list of words' rows included.
//
// W is read once and nothing else is large: 32000 x 512 in bf16 are 33 MB, 6.4 us at the rate of a copy, so what counts is to have
// it on its way at once.  A wave takes 16 words and walks their rows alone, fragments straight from memory into registers, 16 loads of
// 16 bytes per lane in flight; words are the rows of the matrix instruction, positions its columns (from LDS), so that a lane holds four
// consecutive words of one position.  The block's eight waves meet in LDS: one part of the statistics per 128 words.
// (A whole 128-byte line of every row per pair of steps instead of half a line per step: 1 to 2 % slower.)
// fp32: v_mfma_f32_16x16x4, a lane group's four consecutive reduction elements one per instruction, which is free as long as both
// operands agree.
#include <climits>

#include "common.h"
#include "lds_limit.h"
#include "vocab.h"
#include "vocab_epi_dev.h"

namespace asx {
namespace {

typedef uint32_t fu32x4_t __attribute__((ext_vector_type(4)));
constexpr int kFewThreads = 512, kFewWords = kVocabFewCols, kFewMost = 128;   // kFewMost: positions

// 16 bytes of a row of W, KS reduction elements per step of 64 lanes
template <typename TE> struct FewType;
template <> struct FewType<uint16_t> { static constexpr int kVec = 8, kStep = 32; };
template <> struct FewType<float> { static constexpr int kVec = 4, kStep = 16; };

// A vector as it lies in memory, from inside the row, and what makes elements k .. of it, with zeros behind the row: apart, because what is
// done to a load's result where it is asked for waits for it there.
template <typename TE, bool ALIGNED> __device__ __forceinline__ fu32x4_t few_ask(const TE* row, int k, int H) {
  if constexpr (ALIGNED) {   // H % VEC == 0
    return *reinterpret_cast<const fu32x4_t*>(row + (k < H ? k : 0));
  } else {   // H >= 4, rows start on 4 bytes; the last vector of a row from its end
    static_assert(sizeof(TE) == 4, "bf16 rows are whole vectors");
    typedef fu32x4_t __attribute__((aligned(4))) u32x4_on4_t;
    return *reinterpret_cast<const u32x4_on4_t*>(row + (k + 4 <= H ? k : H - 4));
  }
}
template <typename TE, bool ALIGNED> __device__ __forceinline__ fu32x4_t few_fit(const fu32x4_t& x, int k, int H) {
  fu32x4_t q;
  if constexpr (ALIGNED) {
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = k < H ? x[e] : 0u;
  } else {
    const int by = k < H && k + 4 > H ? k + 4 - H : 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t x1 = e + 1 < 4 ? x[e + 1 < 4 ? e + 1 : 3] : 0u, x2 = e + 2 < 4 ? x[e + 2 < 4 ? e + 2 : 3] : 0u, x3 = e == 0 ? x[3] : 0u;
      const uint32_t moved = by == 0 ? x[e] : by == 1 ? x1 : by == 2 ? x2 : x3;
      q[e] = k < H ? moved : 0u;
    }
  }
  return q;
}
template <typename TE, bool ALIGNED> __device__ __forceinline__ fu32x4_t few_load(const TE* row, int k, int H) {
  return few_fit<TE, ALIGNED>(few_ask<TE, ALIGNED>(row, k, H), k, H);
}
template <typename TE> __device__ __forceinline__ f32x4_t few_mul(const fu32x4_t& a, const fu32x4_t& b, f32x4_t acc) {
  if constexpr (sizeof(TE) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
  } else {
    const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], acc, 0, 0, 0);
    return acc;
  }
}

// barrier for LDS alone: the loads of W stay in flight across it
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

// Words' rows 16 NJ y on (row_blocks of them), kc columns of them in LDS at a time: all, or kFewSteps steps, which is a pass over W less than
// fewer rows with all of theirs.  Dynamic LDS: 16 NJ rows of ldk elements of TE, with a teacher 16 NJ rows of kDlLd floats at least.
// The row blocks of the same words follow each other on one XCD: the second one finds W in its L2.
// With a teacher the list and its rows are there already.
constexpr int kDlLd = 132;   // floats of a row in LDS of what there is per word: 128 words
template <typename TE, bool ALIGNED, int NJ, bool ARG, bool TEACH>
__global__ __launch_bounds__(kFewThreads) void vocab_few_kernel(VocabRows p, VocabEpi e, const TE* __restrict__ W, int ldk, int kc, int row_blocks) {
  constexpr int VEC = FewType<TE>::kVec, STEP = FewType<TE>::kStep, U = 8, ROWS = 16 * NJ;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int from[kFewMost], word[kFewMost], count;
  __shared__ float sm[8][ROWS], ss[8][ROWS], st[8][TEACH ? ROWS : 1];
  __shared__ int si[8][ROWS];
  TE* hs = reinterpret_cast<TE*>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, c = lane & 15;
  const int H = p.H, nk = (H + STEP - 1) / STEP;
  const int words = (p.V + kFewWords - 1) / kFewWords, slot = blockIdx.x >> 3;
  const int xb = row_blocks == 1 ? (int)blockIdx.x : slot / row_blocks * 8 + (blockIdx.x & 7), yb = row_blocks == 1 ? 0 : slot % row_blocks;
  if (xb >= words) return;
  const int v0 = xb * kFewWords + wave * 16;
  const TE* row = W + (int64_t)(v0 + c < p.V ? v0 + c : p.V - 1) * H;   // words outside repeat the last one
  fu32x4_t wa[U], wb[U];
  auto load = [&](fu32x4_t (&w)[U], int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = few_ask<TE, ALIGNED>(row, (s0 + u) * STEP + q * VEC, H);
  };
  int y_lane[kFewMost / 64];
#pragma unroll
  for (int k = 0; k < kFewMost / 64; ++k) y_lane[k] = lane + 64 * k < p.N ? p.targets[lane + 64 * k] : -1;
  load(wa, 0);
  load(wb, U);
  if (wave == 0) {   // the words among the positions, in order
    int before = 0;
#pragma unroll
    for (int k = 0; k < kFewMost / 64; ++k) {
      const int n = lane + 64 * k, y = y_lane[k];
      const bool in = n < p.N, is = in && y >= 0 && y < p.V && y != p.pad_id;
      const uint64_t m = __ballot(is);
      const int r = before + __popcll(m & ((1ull << lane) - 1));
      before += __popcll(m);
      if (is) {
        from[r] = n;
        word[r] = y;
      }
      if (!TEACH && xb == 0 && yb == 0) {
        if (in) p.row_pos[n] = is ? r : -1;
        if (is) {
          p.rows[r] = n;
          p.y[r] = y;
        } else if (in) {
          if (p.tok_loss) p.tok_loss[n] = 0.f;
          if (p.argmax) p.argmax[n] = p.pad_id;
        }
      }
    }
    if (lane == 0) {
      count = before;
      if (!TEACH && xb == 0 && yb == 0) {
        *p.n_act = before;
        *p.ticket = 0;
      }
    }
  }
  lds_barrier();
  const int r0 = yb * ROWS, R = count - r0 < ROWS ? count - r0 : ROWS;   // this block's rows
  if (R <= 0) return;
  auto columns = [&](int k0) {   // of the rows to LDS, and as the backward pass wants them, a block each
    const int vecs = kc / VEC;
    for (int i = tid; i < ROWS * vecs; i += kFewThreads) {
      const int r = i / vecs, k = (i - r * vecs) * VEC;
      fu32x4_t x = {0u, 0u, 0u, 0u};
      if (r < R && k0 + k < H) x = few_load<TE, ALIGNED>(reinterpret_cast<const TE*>(p.h) + (int64_t)from[r0 + r] * H, k0 + k, H);
      *reinterpret_cast<fu32x4_t*>(hs + r * ldk + k) = x;
    }
    lds_barrier();
    const int end = k0 + kc < p.ldH ? kc : (int)p.ldH - k0;
    for (int r = TEACH ? R : xb; r < R; r += words) {
      for (int k = tid; k < end; k += kFewThreads) {
        uint16_t* out = p.hc + (int64_t)(r0 + r) * p.ldH + k0 + k;
        if constexpr (sizeof(TE) == 2) {
          *out = hs[r * ldk + k];
        } else {
          float x = hs[r * ldk + k];
#pragma unroll
          for (int t = 0; t < 3; ++t) out[t * p.plane] = (uint16_t)bf16_term(x);
        }
      }
    }
  };
  columns(0);
  f32x4_t acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  int first = 0;   // step that LDS begins with
  auto mul = [&](fu32x4_t (&w)[U], int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u;
      if (s >= nk) continue;
      if ((s + 1) * STEP > H) w[u] = few_fit<TE, ALIGNED>(w[u], s * STEP + q * VEC, H);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        acc[j] = few_mul<TE>(w[u], *reinterpret_cast<const fu32x4_t*>(hs + (16 * j + c) * ldk + (s - first) * STEP + q * VEC), acc[j]);
    }
  };
  for (int s0 = 0; s0 < nk; s0 += 2 * U) {
    if ((s0 - first) * STEP == kc) {
      lds_barrier();   // all waves are through with these columns
      first = s0;
      columns(s0 * STEP);
    }
    mul(wa, s0);
    if (s0 + 2 * U < nk) load(wa, s0 + 2 * U);
    mul(wb, s0 + U);
    if (s0 + 3 * U < nk) load(wb, s0 + 3 * U);
  }
  constexpr float L2E = 1.4426950408889634f;
  const float scale_t = L2E * e.inv_tau;
  float* stage = reinterpret_cast<float*>(smem);
  if constexpr (TEACH) __syncthreads();   // hs has been read
#pragma unroll
  for (int j = 0; j < NJ; ++j) {   // lane: words v0 + 4 q .. + 3 of position 16 j + c
    float x[4], m = -INFINITY;
    const int n = 16 * j + c, y = n < R ? word[r0 + n] - v0 - 4 * q : -1;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int v = v0 + 4 * q + r;
      x[r] = v < p.V ? acc[j][r] + vocab_bias(e, v) : -INFINITY;
      if (r == y) e.at_word[r0 + n] = x[r];
      m = fmaxf(m, x[r]);
    }
    if constexpr (TEACH) *reinterpret_cast<f32x4_t*>(stage + n * kDlLd + wave * 16 + 4 * q) = f32x4_t{x[0], x[1], x[2], x[3]};
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float mb = m > -INFINITY ? m : 0.f;
    float s = 0.f, t = 0.f;
    int idx = INT_MAX;
#pragma unroll
    for (int r = 3; r >= 0; --r) {
      s += __builtin_amdgcn_exp2f((x[r] - mb) * L2E);
      if constexpr (TEACH) t += __builtin_amdgcn_exp2f((x[r] - mb) * scale_t);
      if constexpr (ARG) idx = x[r] == m ? v0 + 4 * q + r : idx;
    }
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if constexpr (TEACH) {
      t += __shfl_xor(t, 16, 64);
      t += __shfl_xor(t, 32, 64);
    }
    if constexpr (ARG) {
      int o = __shfl_xor(idx, 16, 64);
      idx = o < idx ? o : idx;
      o = __shfl_xor(idx, 32, 64);
      idx = o < idx ? o : idx;
    }
    if (q == 0) {
      sm[wave][n] = m;
      ss[wave][n] = s;
      if constexpr (TEACH) st[wave][n] = t;
      if constexpr (ARG) si[wave][n] = m > -INFINITY ? idx : INT_MAX;
    }
  }
  __syncthreads();
  if constexpr (TEACH) {   // logits of the entries: strips of 64 words, a wave per strip and group of rows
    for (int i = wave; i < 2 * NJ; i += 8) {
      const int g = r0 / kVocabGroup + (i >> 1), strip = xb * (kFewWords / kVocabStrip) + (i & 1);
      if (16 * (i >> 1) >= R || strip >= e.strips) continue;
      const int32_t* runs = e.runs + (int64_t)g * (e.strips + 1) + strip;
      const int end = runs[1];
      for (int k = runs[0] + lane; k < end; k += 64) {
        const uint32_t w = e.ent[k];
        e.ent_l[k] = stage[(16 * (i >> 1) + (int)(w & 15)) * kDlLd + (int)(w >> 4) - xb * kFewWords];
      }
    }
  }
  if (tid >= R) return;
  float m = sm[0][tid];
#pragma unroll
  for (int w = 1; w < 8; ++w) m = fmaxf(m, sm[w][tid]);
  const float mb = m > -INFINITY ? m : 0.f;
  float s = 0.f, t = 0.f;
  int idx = INT_MAX;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    const float d = sm[w][tid] - mb;
    s += ss[w][tid] * __builtin_amdgcn_exp2f(d * L2E);
    if constexpr (TEACH) t += st[w][tid] * __builtin_amdgcn_exp2f(d * scale_t);
    if constexpr (ARG) idx = sm[w][tid] == m && si[w][tid] < idx ? si[w][tid] : idx;
  }
  const int64_t at = (int64_t)xb * e.ldr + r0 + tid;
  e.stat[at] = make_float2(m, s);
  if constexpr (TEACH) e.stat_tau[at] = t;
  if constexpr (ARG) e.stat_idx[at] = idx;
}

constexpr size_t kFewLds = 144 * 1024, kFewLdsBf16 = 80 * 1024;
constexpr int kFewSteps = 32;   // a multiple of the loop's 16
// columns of nj tiles of rows in LDS at a time: whole steps; a row of it has 16 bytes more, which put 16 rows at one k into different banks
int few_columns(int nj, int H, bool f32) {
  const int step = f32 ? 16 : 32, all = (H + step - 1) / step * step;
  const size_t e = f32 ? 4 : 2;
  return (size_t)16 * nj * (all * e + 16) <= (f32 ? kFewLds : kFewLdsBf16) ? all : kFewSteps * step;
}
template <typename TE, bool ALIGNED, int NJ, bool ARG, bool TEACH>
hipError_t launch_few(const VocabRows& p, const VocabEpi& e, const void* W, hipStream_t st) {
  auto kfn = vocab_few_kernel<TE, ALIGNED, NJ, ARG, TEACH>;
  static LdsLimit limit;
  const hipError_t rc = limit.raise(reinterpret_cast<const void*>(kfn), kFewLds);
  if (rc != hipSuccess) return rc;
  const int kc = few_columns(NJ, p.H, sizeof(TE) == 4), ldk = kc + FewType<TE>::kVec, words = (p.V + kFewWords - 1) / kFewWords, row_blocks = (p.N + 16 * NJ - 1) / (16 * NJ);
  size_t smem = (size_t)16 * NJ * ldk * sizeof(TE);
  if (TEACH && smem < (size_t)16 * NJ * kDlLd * 4) smem = (size_t)16 * NJ * kDlLd * 4;
  const int blocks = row_blocks == 1 ? words : (words + 7) / 8 * 8 * row_blocks;
  hipLaunchKernelGGL(kfn, dim3(blocks), dim3(kFewThreads), smem, st, p, e, reinterpret_cast<const TE*>(W), ldk, kc, row_blocks);
  return hipGetLastError();
}
template <typename TE, bool ALIGNED, int NJ>
hipError_t launch_few_rows(const VocabRows& p, const VocabEpi& e, const void* W, bool arg, bool teacher, hipStream_t st) {
  if constexpr (sizeof(TE) == 4)
    if (teacher) return launch_few<TE, ALIGNED, NJ, false, true>(p, e, W, st);
  return arg ? launch_few<TE, ALIGNED, NJ, true, false>(p, e, W, st) : launch_few<TE, ALIGNED, NJ, false, false>(p, e, W, st);
}
template <typename TE, bool ALIGNED>
hipError_t launch_few_of(const VocabRows& p, const VocabEpi& e, const void* W, bool arg, bool teacher, hipStream_t st) {
  const int tiles = (p.N + 15) / 16, blocks = (tiles + 3) / 4, nj = (tiles + blocks - 1) / blocks;   // up to four tiles of 16 rows per block, as many in each
  if (nj == 1) return launch_few_rows<TE, ALIGNED, 1>(p, e, W, arg, teacher, st);
  if (nj == 2) return launch_few_rows<TE, ALIGNED, 2>(p, e, W, arg, teacher, st);
  if constexpr (sizeof(TE) == 4)
    return nj == 3 ? launch_few_rows<TE, ALIGNED, 3>(p, e, W, arg, teacher, st) : launch_few_rows<TE, ALIGNED, 4>(p, e, W, arg, teacher, st);
  return hipErrorInvalidValue;
}

// ---- backward ------------------------------------------------------------------------
// All of it in one pass over W: W is read from memory once, dW written once, and dh leaves as one partial sum per block.  A block owns
// a run of words, 16 per wave at a time.  With dl in fp32 the products are fp32 ones on v_mfma_f32_16x16x4 (no terms), whose rate does
// for a few rows: three products of 16 rows x 128 words x 1024 are 21 us of a compute unit, their bytes 26 to 52.
//   1. logits of 16 words x the rows, W's fragments straight from memory: lane (q, c) holds positions 4 q + r of word c;
//   2. dl in place, db (all rows are here), and dW^T = h^T dl: the registers are the second operand as they lie, instruction r taking
//      positions 4 q + r, and a lane's results are four columns of its word;
//   3. dl through LDS to all waves, each of which owns an eighth of the columns: dh^T += W^T dl^T, W again, from the L2.
struct FewBwd {
  const uint16_t* hc;    // rows of words, one or three planes
  int64_t ldH, plane;
  const int32_t *n_act, *y;
  const float *lse, *lse_tau;
  int N, H, V, ldk;
  const void *W, *bias;
  float a1, a2, inv_tau;
  const int32_t* runs;   // teacher
  const uint32_t* ent;
  const float* ent_p;
  int strips;
  void *dW, *db;
  float* dh_part;        // [block][16 NJ][ldH]
};

// Four columns of a row, as they lie and as floats (columns behind H are not used: of any value, but not out of the row)
template <typename TE> struct Four { using type = fu32x4_t; };
template <> struct Four<uint16_t> { using type = uint2; };
template <typename TE, bool ALIGNED> __device__ __forceinline__ typename Four<TE>::type few_ask4(const TE* row, int k, int H) {
  if constexpr (sizeof(TE) == 2) return *reinterpret_cast<const uint2*>(row + (k < H ? k : 0));   // H % 8 == 0
  else return few_ask<float, ALIGNED>(row, k, H);
}
template <typename TE, bool ALIGNED> __device__ __forceinline__ void few_get4(const typename Four<TE>::type& q0, int k, int H, float (&x)[4]) {
  if constexpr (sizeof(TE) == 2) {
    x[0] = lo_bf16(q0.x);
    x[1] = hi_bf16(q0.x);
    x[2] = lo_bf16(q0.y);
    x[3] = hi_bf16(q0.y);
  } else {
    const fu32x4_t q = ALIGNED ? q0 : few_fit<float, ALIGNED>(q0, k, H);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t w = q[e];
      x[e] = __builtin_bit_cast(float, w);
    }
  }
}

template <typename TE, bool ALIGNED, typename TG, int NJ, int G, bool TEACH>
__global__ __launch_bounds__(kFewThreads) void vocab_few_bwd_kernel(FewBwd p) {
  constexpr int VEC = FewType<TE>::kVec, STEP = FewType<TE>::kStep, U = 8, ROWS = 16 * NJ;
  constexpr float L2E = 1.4426950408889634f;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float s_lse[ROWS], s_lt[ROWS];
  __shared__ int s_y[ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, c = lane & 15;
  const int H = p.H, ldk = p.ldk, nk = (H + STEP - 1) / STEP;
  float* hs = reinterpret_cast<float*>(smem);
  float* dlt = hs + ROWS * ldk;
  const TE* W = reinterpret_cast<const TE*>(p.W);
  const int groups = (p.V + 15) / 16;
  const int g0 = (int)((int64_t)blockIdx.x * groups / gridDim.x), g1 = (int)((int64_t)(blockIdx.x + 1) * groups / gridDim.x);
  fu32x4_t wa[U], wb[U];
  const TE* row = W;
  auto load = [&](fu32x4_t (&w)[U], int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = few_ask<TE, ALIGNED>(row, (s0 + u) * STEP + q * VEC, H);
  };
  auto first_loads = [&](int g) {
    const int v = g * 16 + c;
    row = W + (int64_t)(v < p.V ? v : p.V - 1) * H;
    load(wa, 0);
    load(wb, U);
  };
  if (g0 + wave < g1) first_loads(g0 + wave);
  const int count = *p.n_act, R = count < 0 ? 0 : (count < p.N ? count : p.N);
  for (int i = tid; i < ROWS * (ldk / 4); i += kFewThreads) {
    const int r = i / (ldk / 4), k = (i - r * (ldk / 4)) * 4;
    f32x4_t x = {0.f, 0.f, 0.f, 0.f};
    if (r < R && k < (int)p.ldH) {   // (ldH % 8 == 0)
#pragma unroll
      for (int t = (sizeof(TE) == 2 ? 0 : 2); t >= 0; --t) {
        const uint2 h = *reinterpret_cast<const uint2*>(p.hc + t * p.plane + (int64_t)r * p.ldH + k);
        x += f32x4_t{lo_bf16(h.x), hi_bf16(h.x), lo_bf16(h.y), hi_bf16(h.y)};   // (exact: the terms of one fp32 value)
      }
    }
    *reinterpret_cast<f32x4_t*>(hs + r * ldk + k) = x;
  }
  if (tid < ROWS) {
    s_lse[tid] = tid < R ? p.lse[tid] : 0.f;
    s_y[tid] = tid < R ? p.y[tid] : -1;
    if (TEACH) s_lt[tid] = tid < R ? p.lse_tau[tid] : INFINITY;
  }
  lds_barrier();
  f32x4_t dh[NJ][G][4];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) dh[j][g][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int base = g0; base < g1; base += 8) {
    const int v0 = (base + wave) * 16;
    if (base + wave < g1) {
      // 1. logits: positions are the rows, words the columns
      f32x4_t acc[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      auto mul = [&](fu32x4_t (&w)[U], int s0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (s0 + u >= nk) continue;
          if ((s0 + u + 1) * STEP > H) w[u] = few_fit<TE, ALIGNED>(w[u], (s0 + u) * STEP + q * VEC, H);
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            const float* h = hs + (16 * j + c) * ldk + (s0 + u) * STEP + q * VEC;
            const f32x4_t h0 = *reinterpret_cast<const f32x4_t*>(h);
            if constexpr (sizeof(TE) == 2) {
              const f32x4_t h1 = *reinterpret_cast<const f32x4_t*>(h + 4);
              const fu32x4_t b = {pack_bf16(h0[0], h0[1]), pack_bf16(h0[2], h0[3]), pack_bf16(h1[0], h1[1]), pack_bf16(h1[2], h1[3])};   // exact
              acc[j] = few_mul<TE>(b, w[u], acc[j]);
            } else {
              acc[j] = few_mul<TE>(__builtin_bit_cast(fu32x4_t, h0), w[u], acc[j]);
            }
          }
        }
      };
      for (int s0 = 0; s0 < nk; s0 += 2 * U) {
        mul(wa, s0);
        if (s0 + 2 * U < nk) load(wa, s0 + 2 * U);
        mul(wb, s0 + U);
        if (s0 + 3 * U < nk) load(wb, s0 + 3 * U);
      }
      // 2. dl of positions 16 j + 4 q + r, word v0 + c
      const int v = v0 + c;
      const bool in = v < p.V;
      float b = 0.f;
      if (in && p.bias) b = sizeof(TE) == 4 ? reinterpret_cast<const float*>(p.bias)[v] : bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p.bias)[v]);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int n = 16 * j + 4 * q + r;
          const float l = acc[j][r] + b;
          const RowExp e1(s_lse[n]);
          float d = p.a1 * (e1.k * e1(l, L2E) - (s_y[n] == v ? 1.f : 0.f));
          if constexpr (TEACH) {
            const RowExp et(s_lt[n]);
            d += p.a2 * (et.k * et(l, L2E * p.inv_tau));
          }
          acc[j][r] = in && n < R ? d : 0.f;
          dlt[n * kDlLd + wave * 16 + c] = acc[j][r];
        }
      }
      if constexpr (TEACH) {   // this wave's words' entries
        __builtin_amdgcn_s_waitcnt(0xC07F);
        const int strip = v0 / kVocabStrip;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if (16 * j >= R) continue;
          const int32_t* runs = p.runs + (int64_t)j * (p.strips + 1) + strip;
          const int end = runs[1];
          for (int k = runs[0] + lane; k < end; k += 64) {
            const uint32_t w = p.ent[k];
            const int word = (int)(w >> 4) - v0;
            if (word >= 0 && word < 16) dlt[(16 * j + (w & 15)) * kDlLd + wave * 16 + word] -= p.a2 * p.ent_p[k];
          }
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[j][r] = dlt[(16 * j + 4 * q + r) * kDlLd + wave * 16 + c];
      }
      if (p.db) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) sum += (acc[j][0] + acc[j][1]) + (acc[j][2] + acc[j][3]);
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (q == 0 && in) st_elem<TG>(reinterpret_cast<TG*>(p.db), v, sum);
      }
      // dW: two tiles of 16 columns, row i of tile t being column 8 (i / 4) + 4 t + i % 4 for bf16 (a lane then has eight in a row)
      TG* out = reinterpret_cast<TG*>(p.dW) + (int64_t)v * H;
#pragma unroll 1
      for (int k0 = 0; k0 < H; k0 += 32) {
        f32x4_t d[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
        float h[2][NJ][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int col = k0 + (sizeof(TG) == 2 ? 8 * (c >> 2) + 4 * t + (c & 3) : 16 * t + c);
#pragma unroll
          for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) h[t][j][r] = hs[(16 * j + 4 * q + r) * ldk + col];
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int t = 0; t < 2; ++t) d[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(h[t][j][r], acc[j][r], d[t], 0, 0, 0);
        if (!in) continue;
        if constexpr (sizeof(TG) == 2) {
          if (k0 + 8 * q < H)
            *reinterpret_cast<uint4*>(out + k0 + 8 * q) =
                make_uint4(pack_bf16(d[0][0], d[0][1]), pack_bf16(d[0][2], d[0][3]), pack_bf16(d[1][0], d[1][1]), pack_bf16(d[1][2], d[1][3]));
        } else {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int col = k0 + 16 * t + 4 * q;
            if constexpr (ALIGNED) {
              if (col < H) *reinterpret_cast<f32x4_t*>(out + col) = d[t];
            } else if (col + 4 <= H) {
              typedef f32x4_t __attribute__((aligned(4))) f32x4_on4_t;
              *reinterpret_cast<f32x4_on4_t*>(out + col) = d[t];
            } else {
#pragma unroll
              for (int e = 0; e < 3; ++e)
                if (col + e < H) out[col + e] = d[t][e];
            }
          }
        }
      }
    }
    if (base + 8 + wave < g1) first_loads(base + 8 + wave);   // of the next words, while the others' are multiplied
    lds_barrier();
    // 3. this wave's columns: 64 G from 64 G wave on, column 4 i + e of a group being row i of tile e
    constexpr int AHEAD = G * NJ <= 2 ? 2 : 1;   // words' values asked for while the ones ahead are multiplied, where registers allow
    typename Four<TE>::type w[AHEAD][G][4];
    auto ask = [&](int i, typename Four<TE>::type (&x)[G][4]) {
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int v = (base + i) * 16 + 4 * q + r;
          x[g][r] = few_ask4<TE, ALIGNED>(W + (int64_t)(v < p.V ? v : p.V - 1) * H, (wave * G + g) * 64 + 4 * c, H);
        }
    };
    auto times = [&](int i, const typename Four<TE>::type (&x)[G][4]) {
      f32x4_t dl[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) dl[j] = *reinterpret_cast<const f32x4_t*>(dlt + (16 * j + c) * kDlLd + 16 * i + 4 * q);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float f[4];
          few_get4<TE, ALIGNED>(x[g][r], (wave * G + g) * 64 + 4 * c, H, f);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < NJ; ++j) dh[j][g][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[e], dl[j][r], dh[j][g][e], 0, 0, 0);
        }
    };
    if (wave * G * 64 < H) {
      const int n = g1 - base < 8 ? g1 - base : 8;
      if constexpr (AHEAD == 2) {
        ask(0, w[0]);
#pragma unroll 1
        for (int i = 0; i < n; i += 2) {
          if (i + 1 < n) ask(i + 1, w[1]);
          times(i, w[0]);
          if (i + 2 < n) ask(i + 2, w[0]);
          if (i + 1 < n) times(i + 1, w[1]);
        }
      } else {
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
          ask(i, w[0]);
          times(i, w[0]);
        }
      }
    }
    lds_barrier();   // dl has been read
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int n = 16 * j + c;
    if (n >= R) continue;
    float* out = p.dh_part + ((int64_t)blockIdx.x * ROWS + n) * p.ldH;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int col = (wave * G + g) * 64 + 16 * q + 4 * r;
        if (col < (int)p.ldH) *reinterpret_cast<f32x4_t*>(out + col) = f32x4_t{dh[j][g][0][r], dh[j][g][1][r], dh[j][g][2][r], dh[j][g][3][r]};
      }
  }
}

// dh[n]: the blocks' parts, 16 phases of every 16th, eight together, the phases in order; 64 columns of a position per block
template <typename TG>
__global__ __launch_bounds__(256) void vocab_few_dh_kernel(const float* __restrict__ part, int parts, int rows, int64_t ldH,
                                                           const int32_t* __restrict__ row_pos, int H, TG* __restrict__ dh) {
  __shared__ f32x4_t red[16][16];
  const int n = blockIdx.y, at = row_pos[n], r = at < rows ? at : -1, t = threadIdx.x & 15, phase = threadIdx.x >> 4, col = blockIdx.x * 64 + 4 * t;
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  if (r >= 0 && col < (int)ldH) {
    const float* from = part + (int64_t)r * ldH + col;
    const int64_t step = (int64_t)rows * ldH;
#pragma unroll 8
    for (int i = phase; i < parts; i += 16) s += *reinterpret_cast<const f32x4_t*>(from + i * step);
  }
  red[phase][t] = s;
  __syncthreads();
  if (phase != 0) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) s += red[k][t];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (col + e < H) st_elem<TG>(dh + (int64_t)n * H, col + e, s[e]);
}

// tiles of 16 rows and groups of 64 columns per wave of the backward kernel: registers for 4 of their products, LDS
int few_bwd_ldk(int H) { return (H + 31) / 32 * 32 + 4; }
size_t few_bwd_lds(int nj, int H) { return (size_t)16 * nj * (few_bwd_ldk(H) + kDlLd) * 4; }
int few_bwd_groups(int H) {
  const int g = (H + 511) / 512;
  return g <= 2 ? g : 4;
}
int few_bwd_blocks(int V) {   // small vocabularies over the whole chip too: 32 words per block
  const int b = (V + 31) / 32;
  return b < 256 ? b : 256;
}
template <typename TE, bool ALIGNED, typename TG, int NJ, int G, bool TEACH> hipError_t launch_few_bwd(const FewBwd& p, hipStream_t st) {
  auto kfn = vocab_few_bwd_kernel<TE, ALIGNED, TG, NJ, G, TEACH>;
  const int smem = (int)few_bwd_lds(NJ, p.H);
  static LdsLimit limit;
  const hipError_t rc = limit.raise(reinterpret_cast<const void*>(kfn), 156 * 1024);
  if (rc != hipSuccess) return rc;
  hipLaunchKernelGGL(kfn, dim3(few_bwd_blocks(p.V)), dim3(kFewThreads), smem, st, p);
  return hipGetLastError();
}
template <typename TE, bool ALIGNED, typename TG, bool TEACH> hipError_t launch_few_bwd_of(const FewBwd& p, hipStream_t st) {
  const int nj = (p.N + 15) / 16, g = few_bwd_groups(p.H);
  if (nj == 1 && g == 1) return launch_few_bwd<TE, ALIGNED, TG, 1, 1, TEACH>(p, st);
  if (nj == 1 && g == 2) return launch_few_bwd<TE, ALIGNED, TG, 1, 2, TEACH>(p, st);
  if constexpr (sizeof(TG) == 4) {
    if (nj == 2 && g == 1) return launch_few_bwd<TE, ALIGNED, TG, 2, 1, TEACH>(p, st);
  }
  if (nj == 1 && g == 4) return launch_few_bwd<TE, ALIGNED, TG, 1, 4, TEACH>(p, st);
  if constexpr (sizeof(TE) == 4) {
    if (nj == 2 && g == 2) return launch_few_bwd<TE, ALIGNED, TG, 2, 2, TEACH>(p, st);
    if (nj == 3 && g == 1) return launch_few_bwd<TE, ALIGNED, TG, 3, 1, TEACH>(p, st);
    if (nj == 4 && g == 1) return launch_few_bwd<TE, ALIGNED, TG, 4, 1, TEACH>(p, st);
  }
  return hipErrorInvalidValue;
}
template <typename TE, bool ALIGNED, typename TG> hipError_t launch_few_bwd_any(const FewBwd& p, bool teacher, hipStream_t st) {
  return teacher ? launch_few_bwd_of<TE, ALIGNED, TG, true>(p, st) : launch_few_bwd_of<TE, ALIGNED, TG, false>(p, st);
}

}  // namespace

// us, forward, this / the tile kernels behind the list of rows: bf16 1 x 512 x 32000 16.4 / 18.6 (15 of them the host's), 16 x 2048 x 64000
// 63.0 / 68.1, 32 x 512 x 32000 19.1 / 20.0, 32 x 2048 x 64000 65.7 / 69.5, past the line 33 - / 20.5; fp32, whose tiles want W as bf16 terms
// first, 1 x 1024 x 32000 39.4 / 127, 32 x 512 29.3 / 72.4, 16 x 4096 123 / 587, 128 x 256 38.8 / 46.9, 128 x 1024 120 / 150, 128 x 2048 220 / 397;
// with a teacher 8 x 1024 56.1 / 139, 128 x 1024 142 / 162, 40 x 256 x 4000 35.7 / 35.5.
bool vocab_few_rows(int N, int H, bool f32, bool teacher) {
  return f32 ? N <= kFewMost && H >= 4 : !teacher && N <= 32;
}
hipError_t launch_vocab_few(const VocabRows& p, const VocabEpi& e, const void* W, bool arg, bool teacher, hipStream_t st) {
  if (!vocab_few_rows(p.N, p.H, p.f32, teacher)) return hipErrorInvalidValue;
  if (!p.f32) return launch_few_of<uint16_t, true>(p, e, W, arg, teacher, st);
  return p.H % 4 == 0 ? launch_few_of<float, true>(p, e, W, arg, teacher, st) : launch_few_of<float, false>(p, e, W, arg, teacher, st);
}

// us, forward and backward, this / the tile kernels: fp32, whose tiles want W as bf16 terms, 1 x 512 x 32000 69 / 135, 16 x 1024 x 32000 143 /
// 256, 32 x 1024 x 4000 93.4 / 90.8, 48 x 512 x 32000 116 / 159, 64 x 184 x 112000 184 / 281, 64 x 256 x 4000 56.8 / 56.2; bf16, 16 x 512 x 32000 49.1
// / 57.7, 16 x 184 x 112000 68.5 / 83.1, 16 x 1024 x 32000 82.4 / 91.3, 16 x 2048 x 64000 273 / 298, 16 x 1024 x 4000 50.3 / 42.0, with float
// gradients 53.2 / 66.1, 75.3 / 101, 97.3 / 109, 327 / 386, 50.1 / 43.9, 32 x 512 x 32000 64.9 / 69.9; past the line, bf16 gradients, 32 x 512 x
// 32000 69.6 / 61.1.
bool vocab_few_bwd_rows(int N, int H, int V, bool f32, bool g_bf16) {
  const int nj = (N + 15) / 16, g = few_bwd_groups(H);
  if (H < 4 || H > 2048 || nj * g > 4 || few_bwd_lds(nj, H) > 156 * 1024) return false;
  return f32 || nj == 1 || (nj * g == 2 && !g_bf16);
}
size_t vocab_few_bwd_bytes(int N, int H, int V) {
  const int nj = (N + 15) / 16;
  return (size_t)few_bwd_blocks(V) * 16 * nj * ((H + 7) / 8 * 8) * 4;
}
hipError_t launch_vocab_few_bwd(const VocabFewBwd& q, hipStream_t st) {
  if (!vocab_few_bwd_rows(q.N, q.H, q.V, q.f32, q.g_bf16)) return hipErrorInvalidValue;
  FewBwd p{};
  p.hc = q.hc;
  p.ldH = q.ldH;
  p.plane = q.plane;
  p.n_act = q.n_act;
  p.y = q.epi.y;
  p.lse = q.epi.lse;
  p.lse_tau = q.epi.lse_tau;
  p.N = q.N;
  p.H = q.H;
  p.V = q.V;
  p.ldk = few_bwd_ldk(q.H);
  p.W = q.W;
  p.bias = q.epi.bias;
  p.a1 = q.epi.a1;
  p.a2 = q.epi.a2;
  p.inv_tau = q.epi.inv_tau;
  p.runs = q.epi.runs;
  p.ent = q.epi.ent;
  p.ent_p = q.epi.ent_p;
  p.strips = q.epi.strips;
  p.dW = q.dW;
  p.db = q.db;
  p.dh_part = q.dh_part;
  hipError_t e;
  if (!q.f32) e = q.g_bf16 ? launch_few_bwd_any<uint16_t, true, uint16_t>(p, q.teacher, st) : launch_few_bwd_any<uint16_t, true, float>(p, q.teacher, st);
  else if (q.H % 4 == 0) e = launch_few_bwd_any<float, true, float>(p, q.teacher, st);
  else e = launch_few_bwd_any<float, false, float>(p, q.teacher, st);
  if (e != hipSuccess) return e;
  const int rows = (q.N + 15) / 16 * 16;
  const dim3 grid((unsigned)((q.ldH + 63) / 64), q.N);
  if (q.g_bf16)
    hipLaunchKernelGGL(vocab_few_dh_kernel<uint16_t>, grid, dim3(256), 0, st, q.dh_part, few_bwd_blocks(q.V), rows, q.ldH, q.row_pos, q.H, reinterpret_cast<uint16_t*>(q.dh));
  else
    hipLaunchKernelGGL(vocab_few_dh_kernel<float>, grid, dim3(256), 0, st, q.dh_part, few_bwd_blocks(q.V), rows, q.ldH, q.row_pos, q.H, reinterpret_cast<float*>(q.dh));
  return hipGetLastError();
}

}  // namespace asx
