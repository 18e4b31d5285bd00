// Write-out of the vocabulary products: what all kernels share, and that of the 64 x 64 kernel, from the tile in LDS (with the
// bias); that of the larger tiles is in vocab_wave_dev.h.
#pragma once
#include "common.h"
#include "vocab.h"

namespace asx {

// What sets an instance of a product kernel apart: C's write-out, or the vocabulary's, and its arguments.
struct NoVocabOut {
  static constexpr bool kOn = false;
  struct Args {};
};
template <bool TEACH, bool ARG, int TERMS> struct VocabOut {
  static constexpr bool kOn = true, kTeach = TEACH, kArg = ARG;
  static constexpr int kTerms = TERMS;
  using Args = VocabEpi;
};

__device__ __forceinline__ float vocab_bias(const VocabEpi& e, int col) {
  if (!e.bias) return 0.f;
  return e.bias_f32 ? reinterpret_cast<const float*>(e.bias)[col] : bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(e.bias)[col]);
}
// exp(l scale - lse) = k exp2(fma(l, scale log2 e, c)): one fused multiply-add and one v_exp_f32 per element.  k makes up for the
// rounding of c, which is the same for a whole row (|lse| 2^-24 of all of its probabilities, and of 1 - p where a word is nearly certain).
struct RowExp {
  float c, k;
  __device__ __forceinline__ explicit RowExp(float lse) {
    constexpr float L2E = 1.4426950408889634f, L2E_LO = 1.9259629911266175e-8f, LN2 = 0.6931471805599453f;
    c = -lse * L2E;
    const float lo = __builtin_fmaf(-lse, L2E, -c) - lse * L2E_LO;
    k = c > -INFINITY ? __builtin_fmaf(lo, LN2, 1.f) : 1.f;   // (no entries: lse is +inf)
  }
  __device__ __forceinline__ float operator()(float l, float scale_l2e) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(l, scale_l2e, c)); }
};

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

// Four elements of dl as terms, a plane each.  Three are truncated and hold all 24 bits; two are rounded to nearest and off by 2^-17.
template <int TERMS> __device__ __forceinline__ void put_terms(uint16_t* out, int64_t plane, const f32x4_t& v) {
  if constexpr (TERMS == 2) {
    const uint2 hi = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    *reinterpret_cast<uint2*>(out) = hi;
    *reinterpret_cast<uint2*>(out + plane) =
        make_uint2(pack_bf16(v[0] - lo_bf16(hi.x), v[1] - hi_bf16(hi.x)), pack_bf16(v[2] - lo_bf16(hi.y), v[3] - hi_bf16(hi.y)));
  } else {
    float x[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
      uint32_t b[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) b[c] = bf16_term(x[c]);
      *reinterpret_cast<uint2*>(out + t * plane) = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
    }
  }
}

struct VocabRow {
  int y;            // its word
  float c, ct;      // gradient: lse, and at temperature
};
template <bool TEACH, bool GRAD> __device__ __forceinline__ VocabRow vocab_row(const VocabEpi& e, int row, bool in) {
  VocabRow r = {-1, 0.f, 0.f};
  if (in) {
    r.y = e.y[row];
    if constexpr (GRAD) r.c = e.lse[row];
    if constexpr (GRAD && TEACH) r.ct = e.lse_tau[row];
  }
  return r;
}

// Statistics of the 64 staged rows, four lanes per row (every fourth vector of four columns each); row0: the first row,
// left: rows inside, ncols: columns inside.
template <bool TEACH, bool ARG>
__device__ __forceinline__ void vocab_stats64(const VocabEpi& e, const float* stage, int LD, const VocabRow* rows, int row0, int left,
                                              int n0, int ncols) {
  constexpr int BM = 64, NV = BM / 16, XOR1 = 0xB1, XOR2 = 0x4E;
  constexpr float L2E = 1.4426950408889634f;
  const int tid = threadIdx.x, r = tid >> 2, part = tid & 3;
  const float* row = stage + r * LD;
  f32x4_t x[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) x[i] = *reinterpret_cast<const f32x4_t*>(row + (part + 4 * i) * 4);
  if (ncols < BM) {   // the vocabulary's last tile
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if ((part + 4 * i) * 4 + c >= ncols) x[i][c] = -INFINITY;
  }
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    m = fmaxf(fmaxf(m, x[i][0]), x[i][1]);
    m = fmaxf(fmaxf(m, x[i][2]), x[i][3]);
  }
  m = fmaxf(m, dpp_f<XOR1>(m));
  m = fmaxf(m, dpp_f<XOR2>(m));
  // (the rounding of m log2 e is common to the row's part: |m| 2^-24 on its share of the log-sum-exp)
  const float mb = m > -INFINITY ? -m * L2E : 0.f, scale_t = L2E * e.inv_tau, mbt = m > -INFINITY ? -m * scale_t : 0.f;
  float s0 = 0.f, s1 = 0.f, t0 = 0.f, t1 = 0.f;
  int idx = 0x7fffffff;
#pragma unroll
  for (int i = NV - 1; i >= 0; --i)
#pragma unroll
    for (int c = 3; c >= 0; --c) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][c], L2E, mb));
      if (c & 1) s1 += p;
      else s0 += p;
      if constexpr (TEACH) {
        const float q = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][c], scale_t, mbt));
        if (c & 1) t1 += q;
        else t0 += q;
      }
      if constexpr (ARG) idx = x[i][c] == m ? (part + 4 * i) * 4 + c : idx;
    }
  float s = s0 + s1;
  s += dpp_f<XOR1>(s);
  s += dpp_f<XOR2>(s);
  if constexpr (TEACH) {
    t0 += t1;
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
    const int c = rows[r].y - e.v0 - n0;
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

// dl / alpha of the 64 staged rows; cs: the thread's column sums.  256 threads, BM / 4 per row.
template <bool TEACH, int TERMS>
__device__ __forceinline__ void vocab_grad64(const VocabEpi& e, float* stage, int LD, const VocabRow* rows, int row0, int left, int n0,
                                             int ncols, f32x4_t& cs) {
  constexpr int BM = 64, VPR = BM / 4, RP = 256 / VPR, NR = 64 / RP;
  constexpr float L2E = 1.4426950408889634f;
  const int tid = threadIdx.x, cv = (tid % VPR) * 4, col = n0 + cv;
  const float scale_t = L2E * e.inv_tau;
  auto dl4 = [&](int r) {
    const f32x4_t l = *reinterpret_cast<const f32x4_t*>(stage + r * LD + cv);
    const VocabRow q = rows[r];
    f32x4_t v;
    const RowExp e1(q.c), et(q.ct);
    const float a1 = e.a1 * e1.k, a2 = e.a2 * et.k;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float p = e1(l[c], L2E);
      if constexpr (TEACH) v[c] = a1 * p + a2 * et(l[c], scale_t);
      else v[c] = e1.k * p;
    }
    const int at = q.y - e.v0 - col;
    if ((uint32_t)at < 4u) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c == at) v[c] = TEACH ? v[c] - e.a1 : v[c] - 1.f;
    }
    if (ncols < BM) {
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = cv + c < ncols ? v[c] : 0.f;
    }
    return v;
  };
  auto put = [&](int r, f32x4_t v) {
    cs += v;
    if (col >= e.ldd) return;
    put_terms<TERMS>(e.dl + (int64_t)(row0 + r) * e.ldd + col, e.plane, v);
  };
  if constexpr (!TEACH) {
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      const int r = u * RP + tid / VPR;
      if (r < left) put(r, dl4(r));
    }
  } else {
    // the dense part back into the staged rows, the entries' probabilities off it (each place comes once), then out
#pragma unroll
    for (int u = 0; u < NR; ++u) {
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
        stage[(w * kVocabGroup + (k & 15)) * LD + (int)(k >> 4) - e.v0 - n0] -= e.a2 * e.ent_p[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      const int r = u * RP + tid / VPR;
      if (r < left) put(r, *reinterpret_cast<const f32x4_t*>(stage + r * LD + cv));
    }
  }
}

}  // namespace asx
