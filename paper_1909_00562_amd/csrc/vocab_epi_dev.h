// Write-out of the vocabulary products in the 64 x 64 and 128 x 128 kernel: 64 rows of the tile at a time in LDS (with the bias).
#pragma once
#include "common.h"
#include "vocab.h"

namespace asx {

__device__ __forceinline__ float vocab_bias(const VocabEpi& e, int col) {
  if (!e.bias) return 0.f;
  return e.bias_f32 ? reinterpret_cast<const float*>(e.bias)[col] : bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(e.bias)[col]);
}
// exp(x) with the product by log2 e compensated: its rounding alone is |x| 2^-24, a row's probabilities reach down to e^-30
__device__ __forceinline__ float vocab_exp(float x) {
  constexpr float L2E = 1.4426950408889634f, L2E_LO = 1.9259629911266175e-8f;
  const float t = x * L2E;
  const float lo = __builtin_fmaf(x, L2E, -t) + x * L2E_LO;
  const float r = __builtin_amdgcn_exp2f(t);
  return t > -126.f ? __builtin_fmaf(r, lo * 0.6931471805599453f, r) : r;   // (x = -inf: lo is NaN)
}

template <int CTRL> __device__ __forceinline__ float dpp_f(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
template <int CTRL> __device__ __forceinline__ int dpp_i(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, false); }

// Truncated: no term is infinite where x is not, and what is left after each is exact.
__device__ __forceinline__ uint32_t bf16_term(float& x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x) & 0xffff0000u;
  x -= __builtin_bit_cast(float, b);
  return b >> 16;
}

// Statistics of the 64 staged rows, four lanes per row (every fourth vector of four columns each); row0: the first row,
// left: rows inside, ncols: columns inside.
template <int BM, bool TEACH, bool ARG>
__device__ __forceinline__ void vocab_stats64(const VocabEpi& e, const float* stage, int LD, int row0, int left, int n0, int ncols) {
  constexpr int NV = BM / 16, XOR1 = 0xB1, XOR2 = 0x4E;
  const int tid = threadIdx.x, r = tid >> 2, part = tid & 3;
  const float* row = stage + r * LD;
  f32x4_t x[NV];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    x[i] = *reinterpret_cast<const f32x4_t*>(row + (part + 4 * i) * 4);
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if ((part + 4 * i) * 4 + c >= ncols) x[i][c] = -INFINITY;
    m = fmaxf(fmaxf(m, x[i][0]), x[i][1]);
    m = fmaxf(fmaxf(m, x[i][2]), x[i][3]);
  }
  m = fmaxf(m, dpp_f<XOR1>(m));
  m = fmaxf(m, dpp_f<XOR2>(m));
  const float mb = m > -INFINITY ? m : 0.f;
  float s0 = 0.f, s1 = 0.f, t0 = 0.f;
  int idx = 0x7fffffff;
#pragma unroll
  for (int i = NV - 1; i >= 0; --i)
#pragma unroll
    for (int c = 3; c >= 0; --c) {
      const float d = (x[i][c] - mb) * 1.4426950408889634f;
      const float p = __builtin_amdgcn_exp2f(d);
      if (c & 1) s1 += p;
      else s0 += p;
      if constexpr (TEACH) t0 += __builtin_amdgcn_exp2f(d * e.inv_tau);
      if constexpr (ARG) idx = x[i][c] == m ? (part + 4 * i) * 4 + c : idx;
    }
  float s = s0 + s1;
  s += dpp_f<XOR1>(s);
  s += dpp_f<XOR2>(s);
  if constexpr (TEACH) {
    t0 += dpp_f<XOR1>(t0);
    t0 += dpp_f<XOR2>(t0);
  }
  if constexpr (ARG) {
    int o = dpp_i<XOR1>(idx);
    idx = o < idx ? o : idx;
    o = dpp_i<XOR2>(idx);
    idx = o < idx ? o : idx;
  }
  if (part == 0 && r < left) {
    const int64_t at = (int64_t)(n0 / BM) * e.ldr + row0 + r;
    e.stat[at] = make_float2(m, s);
    if constexpr (TEACH) e.stat_tau[at] = t0;
    if constexpr (ARG) e.stat_idx[at] = idx < ncols && m > -INFINITY ? e.v0 + n0 + idx : 0x7fffffff;
    const int c = e.y[row0 + r] - e.v0 - n0;
    if (c >= 0 && c < BM && c < ncols) e.at_word[row0 + r] = row[c];
  }
  if constexpr (TEACH) {   // a wave per group of 16 rows
    const int w = tid >> 6;
    if (w * kVocabGroup < left) {
      const int32_t* runs = e.runs + (int64_t)(row0 / kVocabGroup + w) * (e.strips + 1);
      const int s0i = (e.v0 + n0) / kVocabStrip, s1i = s0i + BM / kVocabStrip < e.strips ? s0i + BM / kVocabStrip : e.strips;
      for (int i = runs[s0i] + (tid & 63); i < runs[s1i]; i += 64) {
        const uint32_t k = e.ent[i];
        e.ent_l[i] = stage[(w * kVocabGroup + (k & 15)) * LD + (int)(k >> 4) - e.v0 - n0];
      }
    }
  }
}

// dl of the 64 staged rows; cs: the thread's column sums.  256 threads, BM / 4 per row.
template <int BM, bool TEACH, int TERMS>
__device__ __forceinline__ void vocab_grad64(const VocabEpi& e, float* stage, int LD, int row0, int left, int n0, int ncols, f32x4_t& cs) {
  constexpr int VPR = BM / 4, RP = 256 / VPR;
  const int tid = threadIdx.x, cv = (tid % VPR) * 4, col = n0 + cv;
  auto dl4 = [&](int r) {
    f32x4_t v = *reinterpret_cast<const f32x4_t*>(stage + r * LD + cv);
    const float lse = e.lse[row0 + r], lt = TEACH ? e.lse_tau[row0 + r] : 0.f;
    const int at = e.y[row0 + r] - e.v0 - col;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float l = v[c];
      float d = e.g * ((TERMS == 1 ? __expf(l - lse) : vocab_exp(l - lse)) - (c == at ? 1.f : 0.f));
      if constexpr (TEACH) d += e.c2 * (TERMS == 1 ? __expf(l * e.inv_tau - lt) : vocab_exp(l * e.inv_tau - lt));
      v[c] = cv + c < ncols ? d : 0.f;
    }
    return v;
  };
  auto put = [&](int r, f32x4_t v) {
    cs += v;
    if (col >= e.ldd) return;
    uint16_t* out = e.dl + (int64_t)(row0 + r) * e.ldd + col;
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
      uint2 q;
      if constexpr (TERMS == 1) {
        q = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
      } else {
        float x[4] = {v[0], v[1], v[2], v[3]};
        uint32_t b[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          b[c] = bf16_term(x[c]);
          v[c] = x[c];
        }
        q = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
      }
      *reinterpret_cast<uint2*>(out + t * e.plane) = q;
    }
  };
  if constexpr (!TEACH) {
#pragma unroll
    for (int u = 0; u < 64 / RP; ++u) {
      const int r = u * RP + tid / VPR;
      if (r < left) put(r, dl4(r));
    }
  } else {
    // the dense part back into the staged rows, the entries' probabilities off it (each place comes once), then out
#pragma unroll
    for (int u = 0; u < 64 / RP; ++u) {
      const int r = u * RP + tid / VPR;
      if (r < left) *reinterpret_cast<f32x4_t*>(stage + r * LD + cv) = dl4(r);
    }
    __syncthreads();
    const int w = tid >> 6;
    if (w * kVocabGroup < left) {
      const int32_t* runs = e.runs + (int64_t)(row0 / kVocabGroup + w) * (e.strips + 1);
      const int s0i = (e.v0 + n0) / kVocabStrip, s1i = s0i + BM / kVocabStrip < e.strips ? s0i + BM / kVocabStrip : e.strips;
      for (int i = runs[s0i] + (tid & 63); i < runs[s1i]; i += 64) {
        const uint32_t k = e.ent[i];
        stage[(w * kVocabGroup + (k & 15)) * LD + (int)(k >> 4) - e.v0 - n0] -= e.c2 * e.ent_p[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 64 / RP; ++u) {
      const int r = u * RP + tid / VPR;
      if (r < left) put(r, *reinterpret_cast<const f32x4_t*>(stage + r * LD + cv));
    }
  }
}

}  // namespace asx
