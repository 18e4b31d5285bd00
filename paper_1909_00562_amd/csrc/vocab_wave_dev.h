// Write-out of the vocabulary products in the 256 x 256 and 128 x 128 kernels: a wave's 16 TM x 64 part of the tile from its
// accumulators (16 x 16 tiles: register r of lane l is row 4 (l / 16) + r, column l % 16).  Rows of a wave start at multiples of
// 16 TM, columns at multiples of 64: a 16-row tile and the wave's columns are one group and one strip of the teacher's lists.
#pragma once
#include "vocab_epi_dev.h"

namespace asx {

constexpr int kRor8 = 0x128, kRor4 = 0x124, kRor2 = 0x122, kRor1 = 0x121;   // rotations inside 16 lanes
__device__ __forceinline__ float max16(float v) {
  v = fmaxf(v, dpp_f<kRor8>(v));
  v = fmaxf(v, dpp_f<kRor4>(v));
  v = fmaxf(v, dpp_f<kRor2>(v));
  return fmaxf(v, dpp_f<kRor1>(v));
}
__device__ __forceinline__ float sum16(float v) {
  v += dpp_f<kRor8>(v);
  v += dpp_f<kRor4>(v);
  v += dpp_f<kRor2>(v);
  return v + dpp_f<kRor1>(v);
}
__device__ __forceinline__ int min16(int v) {
  auto least = [](int a, int b) { return a < b ? a : b; };
  v = least(v, dpp_i<kRor8>(v));
  v = least(v, dpp_i<kRor4>(v));
  v = least(v, dpp_i<kRor2>(v));
  return least(v, dpp_i<kRor1>(v));
}
// float offset of (row, column) of a staged 16 x 64 part (as the kernel's stage_round writes it)
__device__ __forceinline__ int staged_at(int row, int col) { return row * 64 + ((((col >> 4) ^ (row >> 2)) & 3) << 4) + (col & 15); }
constexpr int kWaitLgkm = 0xC07F;

// The teacher's entries of a wave's 16-row tiles: the bounds of all runs up front, an entry per lane of each one tile ahead
template <int TM> struct WaveEntries {
  int run0[TM], run1[TM];
  uint32_t w;
  float p;
  __device__ __forceinline__ void init(const VocabEpi& e, int row0, int rows_left, int strip) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const bool in = 16 * i < rows_left;
      const int32_t* r = e.runs + (int64_t)(row0 / kVocabGroup + (in ? i : 0)) * (e.strips + 1) + strip;
      run0[i] = r[0];
      run1[i] = in ? r[1] : run0[i];
    }
  }
  template <bool PROB> __device__ __forceinline__ void ask(const VocabEpi& e, int i, int lane) {
    w = 0;
    p = 0.f;
    if (run0[i] + lane < run1[i]) {
      w = e.ent[run0[i] + lane];
      if (PROB) p = e.ent_p[run0[i] + lane];
    }
  }
};

// Softmax statistics, straight from the registers: maximum and sum over a lane's four columns, then over 16 lanes.
template <bool TEACH, bool ARG, int TM, typename Stage>
__device__ __forceinline__ void vocab_wave_stats(const VocabEpi& e, f32x4_t (&acc)[TM][4], float* region, Stage stage, int lane, int row0,
                                                 int rows_left, int col0, int ncols) {
  constexpr float L2E = 1.4426950408889634f;
  const int c = lane & 15, q = lane >> 4, strip = (e.v0 + col0) / kVocabStrip;
  if (rows_left <= 0 || col0 >= ncols) return;
  int4 y[TM];   // (rows behind the last are inside the array's padding)
#pragma unroll
  for (int i = 0; i < TM; ++i) y[i] = *reinterpret_cast<const int4*>(e.y + row0 + 16 * i + 4 * q);
  WaveEntries<TM> entries;
  if constexpr (TEACH) {
    entries.init(e, row0, rows_left, strip);
    entries.template ask<false>(e, 0, lane);
  }
  float bias[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) bias[j] = col0 + 16 * j + c < ncols ? vocab_bias(e, col0 + 16 * j + c) : 0.f;
  const float scale_t = L2E * e.inv_tau;
  const bool ragged = ncols - col0 < 64;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    float m[4], s[4], t[4];
    int best[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = acc[i][j][r] + bias[j];
        if (TEACH) acc[i][j][r] = x[j];
        if (ragged) x[j] = col0 + 16 * j + c < ncols ? x[j] : -INFINITY;
      }
      const int at = (r == 0 ? y[i].x : r == 1 ? y[i].y : r == 2 ? y[i].z : y[i].w) - e.v0 - col0 - c;
      if ((at & ~48) == 0 && 16 * i + 4 * q + r < rows_left)
        e.at_word[row0 + 16 * i + 4 * q + r] = at < 32 ? (at == 0 ? x[0] : x[1]) : (at == 32 ? x[2] : x[3]);
      m[r] = max16(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
      if constexpr (ARG) {
        int b = 0x7fffffff;
#pragma unroll
        for (int j = 3; j >= 0; --j) b = x[j] == m[r] ? 16 * j + c : b;
        best[r] = min16(b);
      }
      const float mb = m[r] > -INFINITY ? -m[r] * L2E : 0.f;
      float p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], L2E, mb));
      s[r] = sum16((p[0] + p[1]) + (p[2] + p[3]));
      if constexpr (TEACH) {
        const float mt = m[r] > -INFINITY ? -m[r] * scale_t : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], scale_t, mt));
        t[r] = sum16((p[0] + p[1]) + (p[2] + p[3]));
      }
    }
    const float m1 = c == 0 ? m[0] : c == 1 ? m[1] : c == 2 ? m[2] : m[3], s1 = c == 0 ? s[0] : c == 1 ? s[1] : c == 2 ? s[2] : s[3];
    if (c < 4 && 16 * i + 4 * q + c < rows_left) {
      const int64_t at = (int64_t)(col0 / 64) * e.ldr + row0 + 16 * i + 4 * q + c;
      e.stat[at] = make_float2(m1, s1);
      if constexpr (ARG) {
        const int b = c == 0 ? best[0] : c == 1 ? best[1] : c == 2 ? best[2] : best[3];
        e.stat_idx[at] = m1 > -INFINITY && b < 64 ? e.v0 + col0 + b : 0x7fffffff;
      }
      if constexpr (TEACH) e.stat_tau[at] = c == 0 ? t[0] : c == 1 ? t[1] : c == 2 ? t[2] : t[3];
    }
    if constexpr (TEACH) {
      const uint32_t w0 = entries.w;
      if (i + 1 < TM) entries.template ask<false>(e, i + 1, lane);
      if (entries.run0[i] < entries.run1[i]) {
        stage(i);
        __builtin_amdgcn_s_waitcnt(kWaitLgkm);
        for (int k = entries.run0[i] + lane; k < entries.run1[i]; k += 64) {
          const uint32_t w = k == entries.run0[i] + lane ? w0 : e.ent[k];
          e.ent_l[k] = region[staged_at(w & 15, (int)(w >> 4) - e.v0 - col0)];
        }
        __builtin_amdgcn_s_waitcnt(kWaitLgkm);
      }
    }
  }
}

// dl / alpha: from the accumulators in place, 16 rows at a time through the wave's slice of LDS, from where the teacher's
// probabilities go off it, the columns are added up and whole row vectors are written.
template <bool TEACH, int TERMS, int TM, typename Stage>
__device__ __forceinline__ void vocab_wave_grad(const VocabEpi& e, f32x4_t (&acc)[TM][4], float* region, Stage stage, int lane, int row0,
                                                int rows_left, int col0, int ncols) {
  constexpr float L2E = 1.4426950408889634f;
  const int c = lane & 15, q = lane >> 4, strip = (e.v0 + col0) / kVocabStrip;
  const int vcol = c * 4;
  if (rows_left <= 0 || col0 >= ncols) return;   // (the teacher's runs end with the last group of rows)
  const float scale_t = L2E * e.inv_tau;
  float bias[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) bias[j] = col0 + 16 * j + c < ncols ? vocab_bias(e, col0 + 16 * j + c) : 0.f;
  const bool ragged = ncols - col0 < 64, last = rows_left < 16 * TM;
  f32x4_t cs = {0.f, 0.f, 0.f, 0.f};
  struct Rows {   // (arrays padded to whole tiles)
    int4 y;
    f32x4_t lse, lt;
  };
  auto rows_of = [&](int i) {   // asked for one tile ahead
    Rows q;
    const int at = row0 + 16 * i + 4 * (lane >> 4);
    q.y = *reinterpret_cast<const int4*>(e.y + at);
    q.lse = *reinterpret_cast<const f32x4_t*>(e.lse + at);
    q.lt = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if constexpr (TEACH) q.lt = *reinterpret_cast<const f32x4_t*>(e.lse_tau + at);
    return q;
  };
  WaveEntries<TM> entries;
  if constexpr (TEACH) {
    entries.init(e, row0, rows_left, strip);
    entries.template ask<true>(e, 0, lane);
  }
  Rows next = rows_of(0);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int4 y = next.y;
    const f32x4_t lse = next.lse, lt = next.lt;
    const uint32_t w0 = entries.w;
    const float p0 = entries.p;
    if (i + 1 < TM) {
      next = rows_of(i + 1);
      if constexpr (TEACH) entries.template ask<true>(e, i + 1, lane);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int at = (r == 0 ? y.x : r == 1 ? y.y : r == 2 ? y.z : y.w) - e.v0 - col0 - c;
      const RowExp e1(lse[r]), et(lt[r]);
      const float a1 = e.a1 * e1.k, a2 = e.a2 * et.k;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float l = acc[i][j][r] + bias[j], p = e1(l, L2E);
        if constexpr (TEACH) acc[i][j][r] = a1 * p + a2 * et(l, scale_t);
        else acc[i][j][r] = e1.k * p;
      }
      if ((at & ~48) == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at == 16 * j) acc[i][j][r] -= TEACH ? e.a1 : 1.f;
      }
      if (ragged || last) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j][r] = col0 + 16 * j + c < ncols && 16 * i + 4 * q + r < rows_left ? acc[i][j][r] : 0.f;
      }
    }
    stage(i);
    __builtin_amdgcn_s_waitcnt(kWaitLgkm);
    if constexpr (TEACH) {
      for (int k = entries.run0[i] + lane; k < entries.run1[i]; k += 64) {
        const bool asked = k == entries.run0[i] + lane;
        const uint32_t w = asked ? w0 : e.ent[k];
        region[staged_at(w & 15, (int)(w >> 4) - e.v0 - col0)] -= e.a2 * (asked ? p0 : e.ent_p[k]);
      }
      __builtin_amdgcn_s_waitcnt(kWaitLgkm);
    }
    f32x4_t v4[4];
#pragma unroll
    for (int it = 0; it < 4; ++it) v4[it] = *reinterpret_cast<const f32x4_t*>(region + staged_at(it * 4 + q, vcol));
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int row = 16 * i + it * 4 + q;
      const f32x4_t v = v4[it];
      cs += v;
      if (row < rows_left && col0 + vcol < e.ldd) put_terms<TERMS>(e.dl + (int64_t)(row0 + row) * e.ldd + col0 + vcol, e.plane, v);
    }
    __builtin_amdgcn_s_waitcnt(kWaitLgkm);   // the slice has been read
  }
  if (e.col_sums) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      cs[k] += __shfl_xor(cs[k], 16, 64);
      cs[k] += __shfl_xor(cs[k], 32, 64);
    }
    if (q == 0) {
      float* out = e.col_sums + (int64_t)(row0 / (16 * TM)) * e.ld_sums + col0 + vcol;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (col0 + vcol + k < ncols) out[k] = cs[k];
    }
  }
}

}  // namespace asx
