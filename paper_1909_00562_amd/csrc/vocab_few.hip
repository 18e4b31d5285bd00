// Few rows (a decoder step): the projection's softmax statistics in one pass over W, the list of words' rows included.
//
// W is read once and nothing else is large: 32000 x 512 in bf16 are 33 MB, 6.4 us at the rate of a copy, so what counts is to have
// it on its way at once.  A wave takes 16 words and walks their rows alone, fragments straight from memory into registers, 16 loads of
// 16 bytes per lane in flight; words are the rows of the matrix instruction, positions its columns (from LDS), so that a lane holds four
// consecutive words of one position.  The block's eight waves meet in LDS: one part of the statistics per 128 words.
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
constexpr int kFewThreads = 512, kFewWords = kVocabFewCols;

// 16 bytes of a row of W, KS reduction elements per step of 64 lanes
template <typename TE> struct FewType;
template <> struct FewType<uint16_t> { static constexpr int kVec = 8, kStep = 32; };
template <> struct FewType<float> { static constexpr int kVec = 4, kStep = 16; };

template <typename TE, bool ALIGNED> __device__ __forceinline__ fu32x4_t few_load(const TE* row, int k, int H) {
  constexpr int VEC = FewType<TE>::kVec;
  if constexpr (ALIGNED) {   // H % VEC == 0
    fu32x4_t q = *reinterpret_cast<const fu32x4_t*>(row + (k < H ? k : 0));
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = k < H ? q[e] : 0u;
    return q;
  } else {
    static_assert(sizeof(TE) == 4, "bf16 rows are whole vectors");
    fu32x4_t q;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float x = row[k + e < H ? k + e : 0];
      q[e] = k + e < H ? __builtin_bit_cast(uint32_t, x) : 0u;
    }
    return q;
  }
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

// Words' rows 16 NJ blockIdx.y on; dynamic LDS: 16 NJ rows of ldk elements of TE
template <typename TE, bool ALIGNED, int NJ, bool ARG>
__global__ __launch_bounds__(kFewThreads) void vocab_few_kernel(VocabRows p, VocabEpi e, const TE* __restrict__ W, int ldk) {
  constexpr int VEC = FewType<TE>::kVec, STEP = FewType<TE>::kStep, U = 8, ROWS = 16 * NJ;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int from[64], word[64], count;
  __shared__ float sm[8][ROWS], ss[8][ROWS];
  __shared__ int si[8][ROWS];
  TE* hs = reinterpret_cast<TE*>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, c = lane & 15;
  const int H = p.H, nk = (H + STEP - 1) / STEP;
  const int v0 = blockIdx.x * kFewWords + wave * 16;
  const TE* row = W + (int64_t)(v0 + c < p.V ? v0 + c : p.V - 1) * H;   // words outside repeat the last one
  fu32x4_t wa[U], wb[U];
  auto load = [&](fu32x4_t (&w)[U], int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = few_load<TE, ALIGNED>(row, (s0 + u) * STEP + q * VEC, H);
  };
  const int y_lane = lane < p.N ? p.targets[lane] : -1;
  load(wa, 0);
  load(wb, U);
  if (wave == 0) {   // the words among the positions (at most 64), in order
    const bool in = lane < p.N;
    const int y = y_lane;
    const bool is = in && y >= 0 && y < p.V && y != p.pad_id;
    const uint64_t m = __ballot(is);
    const int r = __popcll(m & ((1ull << lane) - 1));
    if (is) {
      from[r] = lane;
      word[r] = y;
    }
    if (lane == 0) count = __popcll(m);
    if (blockIdx.x == 0 && blockIdx.y == 0) {
      if (in) p.row_pos[lane] = is ? r : -1;
      if (is) {
        p.rows[r] = lane;
        p.y[r] = y;
      } else if (in) {
        if (p.tok_loss) p.tok_loss[lane] = 0.f;
        if (p.argmax) p.argmax[lane] = p.pad_id;
      }
      if (lane == 0) {
        *p.n_act = __popcll(m);
        *p.ticket = 0;
      }
    }
  }
  lds_barrier();
  const int r0 = blockIdx.y * ROWS, R = count - r0 < ROWS ? count - r0 : ROWS;   // this block's rows
  if (R <= 0) return;
  for (int i = tid; i < ROWS * (ldk / VEC); i += kFewThreads) {
    const int r = i / (ldk / VEC), k = (i - r * (ldk / VEC)) * VEC;
    fu32x4_t x = {0u, 0u, 0u, 0u};
    if (r < R && k < H) x = few_load<TE, ALIGNED>(reinterpret_cast<const TE*>(p.h) + (int64_t)from[r0 + r] * H, k, H);
    *reinterpret_cast<fu32x4_t*>(hs + r * ldk + k) = x;
  }
  lds_barrier();
  for (int r = blockIdx.x; r < R; r += gridDim.x) {   // the rows of words for a backward pass, a block each
    for (int k = tid; k < p.ldH; k += kFewThreads) {
      uint16_t* out = p.hc + (int64_t)(r0 + r) * p.ldH + k;
      if constexpr (sizeof(TE) == 2) {
        *out = hs[r * ldk + k];
      } else {
        float x = hs[r * ldk + k];   // (ldk covers ldH)
#pragma unroll
        for (int t = 0; t < 3; ++t) out[t * p.plane] = (uint16_t)bf16_term(x);
      }
    }
  }
  f32x4_t acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  auto mul = [&](fu32x4_t (&w)[U], int s0) {   // (steps past the end: w is zero, and LDS is read at its last step)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u < nk ? s0 + u : nk - 1;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        acc[j] = few_mul<TE>(w[u], *reinterpret_cast<const fu32x4_t*>(hs + (16 * j + c) * ldk + s * STEP + q * VEC), acc[j]);
    }
  };
  for (int s0 = 0; s0 < nk; s0 += 2 * U) {
    mul(wa, s0);
    if (s0 + 2 * U < nk) load(wa, s0 + 2 * U);
    mul(wb, s0 + U);
    if (s0 + 3 * U < nk) load(wb, s0 + 3 * U);
    else if (s0 + 2 * U < nk) {
#pragma unroll
      for (int u = 0; u < U; ++u) wb[u] = fu32x4_t{0u, 0u, 0u, 0u};
    }
  }
  constexpr float L2E = 1.4426950408889634f;
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
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float mb = m > -INFINITY ? m : 0.f;
    float s = 0.f;
    int idx = INT_MAX;
#pragma unroll
    for (int r = 3; r >= 0; --r) {
      s += __builtin_amdgcn_exp2f((x[r] - mb) * L2E);
      if constexpr (ARG) idx = x[r] == m ? v0 + 4 * q + r : idx;
    }
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if constexpr (ARG) {
      int o = __shfl_xor(idx, 16, 64);
      idx = o < idx ? o : idx;
      o = __shfl_xor(idx, 32, 64);
      idx = o < idx ? o : idx;
    }
    if (q == 0) {
      sm[wave][n] = m;
      ss[wave][n] = s;
      if constexpr (ARG) si[wave][n] = m > -INFINITY ? idx : INT_MAX;
    }
  }
  __syncthreads();
  if (tid >= R) return;
  float m = sm[0][tid];
#pragma unroll
  for (int w = 1; w < 8; ++w) m = fmaxf(m, sm[w][tid]);
  const float mb = m > -INFINITY ? m : 0.f;
  float s = 0.f;
  int idx = INT_MAX;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    s += ss[w][tid] * __builtin_amdgcn_exp2f((sm[w][tid] - mb) * L2E);
    if constexpr (ARG) idx = sm[w][tid] == m && si[w][tid] < idx ? si[w][tid] : idx;
  }
  const int64_t at = (int64_t)blockIdx.x * e.ldr + r0 + tid;
  e.stat[at] = make_float2(m, s);
  if constexpr (ARG) e.stat_idx[at] = idx;
}

constexpr size_t kFewLds = 144 * 1024, kFewLdsBf16 = 80 * 1024;
int few_ldk(int H, bool f32) {   // whole steps, and 16 bytes that put 16 rows at one k into different banks
  const int step = f32 ? 16 : 32;
  return (H + step - 1) / step * step + (f32 ? 4 : 8);
}
template <typename TE, bool ALIGNED, int NJ, bool ARG>
hipError_t launch_few(const VocabRows& p, const VocabEpi& e, const void* W, hipStream_t st) {
  auto kfn = vocab_few_kernel<TE, ALIGNED, NJ, ARG>;
  static LdsLimit limit;
  const hipError_t rc = limit.raise(reinterpret_cast<const void*>(kfn), kFewLds);
  if (rc != hipSuccess) return rc;
  const int ldk = few_ldk(p.H, sizeof(TE) == 4);
  hipLaunchKernelGGL(kfn, dim3((p.V + kFewWords - 1) / kFewWords, (p.N + 16 * NJ - 1) / (16 * NJ)), dim3(kFewThreads), (size_t)16 * NJ * ldk * sizeof(TE), st, p, e,
                     reinterpret_cast<const TE*>(W), ldk);
  return hipGetLastError();
}
// tiles of 16 rows per block: all of them, or as many as fit
int few_tiles(int N, int H, bool f32) {
  const size_t tile = (size_t)16 * few_ldk(H, f32) * (f32 ? 4 : 2), most = f32 ? kFewLds : kFewLdsBf16;
  for (int nj = N <= 16 ? 1 : N <= 32 ? 2 : 4; nj > 0; nj >>= 1)
    if (nj * tile <= most) return nj;
  return 0;
}
template <typename TE, bool ALIGNED>
hipError_t launch_few_of(const VocabRows& p, const VocabEpi& e, const void* W, bool arg, hipStream_t st) {
  const int nj = few_tiles(p.N, p.H, sizeof(TE) == 4);
  if (nj == 1) return arg ? launch_few<TE, ALIGNED, 1, true>(p, e, W, st) : launch_few<TE, ALIGNED, 1, false>(p, e, W, st);
  if (nj == 2) return arg ? launch_few<TE, ALIGNED, 2, true>(p, e, W, st) : launch_few<TE, ALIGNED, 2, false>(p, e, W, st);
  if constexpr (sizeof(TE) == 4) return arg ? launch_few<TE, ALIGNED, 4, true>(p, e, W, st) : launch_few<TE, ALIGNED, 4, false>(p, e, W, st);
  return hipErrorInvalidValue;
}

}  // namespace

// us, forward, this / the tile kernels behind the list of rows: bf16 1 x 512 x 32000 16.4 / 18.6 (15 of them the host's), 16 x 2048 x 64000
// 63.2 / 68.1, 32 x 512 x 32000 19.1 / 20.0, past the line 33 - / 20.5; fp32, whose tiles want W as bf16 terms first, 1 x 1024 x 32000
// 39.4 / 127, 16 x 1024 41.7 / 136, 32 x 512 29.3 / 72.4.
bool vocab_few_rows(int N, int H, bool f32) {
  return f32 ? N <= 64 && few_tiles(N, H, true) > 0 : N <= 32 && 16 * few_tiles(N, H, false) >= N;
}
hipError_t launch_vocab_few(const VocabRows& p, const VocabEpi& e, const void* W, bool arg, hipStream_t st) {
  if (!vocab_few_rows(p.N, p.H, p.f32)) return hipErrorInvalidValue;
  if (!p.f32) return launch_few_of<uint16_t, true>(p, e, W, arg, st);
  return p.H % 4 == 0 ? launch_few_of<float, true>(p, e, W, arg, st) : launch_few_of<float, false>(p, e, W, arg, st);
}

}  // namespace asx
