// Write-out of the vocabulary products in the 256 x 256 kernel: a wave's 128 x 64 part of the tile from its accumulators
// (16 x 16 tiles: register r of lane l is row 4 (l / 16) + r, column l % 16).  Rows of a wave start at multiples of 128, columns at
// multiples of 64: a 16-row tile and the wave's columns are one group and one strip of the teacher's lists.
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
// float offset of (row, column) of a staged 16 x 64 part (as the kernel's stage_round writes it)
__device__ __forceinline__ int staged_at(int row, int col) { return row * 64 + ((((col >> 4) ^ (row >> 2)) & 3) << 4) + (col & 15); }
constexpr int kWaitLgkm = 0xC07F;

// Softmax statistics, straight from the registers: maximum and sum over a lane's four columns, then over 16 lanes.
template <bool TEACH, typename Stage>
__device__ __forceinline__ void vocab_wave_stats(const VocabEpi& e, f32x4_t (&acc)[8][4], float* region, Stage stage, int lane, int row0,
                                                 int rows_left, int col0, int ncols) {
  constexpr float L2E = 1.4426950408889634f;
  const int c = lane & 15, q = lane >> 4, strip = (e.v0 + col0) / kVocabStrip;
  if (rows_left <= 0 || col0 >= ncols) return;
  int4 y[8];   // (rows behind the last are inside the array's padding)
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = *reinterpret_cast<const int4*>(e.y + row0 + 16 * i + 4 * q);
  int run0[8], run1[8];
  if constexpr (TEACH) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool in = 16 * i < rows_left;
      const int32_t* r = e.runs + (int64_t)(row0 / kVocabGroup + (in ? i : 0)) * (e.strips + 1) + strip;
      run0[i] = r[0];
      run1[i] = in ? r[1] : run0[i];
    }
  }
  float bias[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) bias[j] = col0 + 16 * j + c < ncols ? vocab_bias(e, col0 + 16 * j + c) : 0.f;
  const float scale_t = L2E * e.inv_tau;
  const bool ragged = ncols - col0 < 64;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float m[4], s[4], t[4];
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
      if constexpr (TEACH) e.stat_tau[at] = c == 0 ? t[0] : c == 1 ? t[1] : c == 2 ? t[2] : t[3];
    }
    if constexpr (TEACH) {
      if (run0[i] < run1[i]) {
        stage(i);
        __builtin_amdgcn_s_waitcnt(kWaitLgkm);
        for (int k = run0[i] + lane; k < run1[i]; k += 64) {
          const uint32_t w = e.ent[k];
          e.ent_l[k] = region[staged_at(w & 15, (int)(w >> 4) - e.v0 - col0)];
        }
        __builtin_amdgcn_s_waitcnt(kWaitLgkm);
      }
    }
  }
}

// dl / alpha: from the accumulators in place, 16 rows at a time through the wave's slice of LDS, from where the teacher's
// probabilities go off it, the columns are added up and whole row vectors are written.
template <bool TEACH, int TERMS, typename Stage>
__device__ __forceinline__ void vocab_wave_grad(const VocabEpi& e, f32x4_t (&acc)[8][4], float* region, Stage stage, int lane, int row0,
                                                int rows_left, int col0, int ncols) {
  constexpr float L2E = 1.4426950408889634f;
  const int c = lane & 15, q = lane >> 4, strip = (e.v0 + col0) / kVocabStrip;
  const int vcol = c * 4;
  if (col0 >= ncols) return;
  const float scale_t = L2E * e.inv_tau;
  float bias[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) bias[j] = col0 + 16 * j + c < ncols ? vocab_bias(e, col0 + 16 * j + c) : 0.f;
  const bool ragged = ncols - col0 < 64, last = rows_left < 128;
  f32x4_t cs = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int4 y = *reinterpret_cast<const int4*>(e.y + row0 + 16 * i + 4 * q);   // (arrays padded to whole tiles)
    const f32x4_t lse = *reinterpret_cast<const f32x4_t*>(e.lse + row0 + 16 * i + 4 * q);
    f32x4_t lt = {0.f, 0.f, 0.f, 0.f};
    int run0 = 0, run1 = 0;
    if constexpr (TEACH) {
      lt = *reinterpret_cast<const f32x4_t*>(e.lse_tau + row0 + 16 * i + 4 * q);
      if (16 * i < rows_left) {
        const int32_t* r = e.runs + (int64_t)(row0 / kVocabGroup + i) * (e.strips + 1) + strip;
        run0 = r[0];
        run1 = r[1];
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int at = (r == 0 ? y.x : r == 1 ? y.y : r == 2 ? y.z : y.w) - e.v0 - col0 - c;
      const float c1 = -lse[r] * L2E, ct = -lt[r] * L2E;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float l = acc[i][j][r] + bias[j];
        float d = TERMS == 1 ? __builtin_amdgcn_exp2f(__builtin_fmaf(l, L2E, c1)) : vocab_exp(l - lse[r]);
        if constexpr (TEACH) {
          const float dt = TERMS == 1 ? __builtin_amdgcn_exp2f(__builtin_fmaf(l, scale_t, ct)) : vocab_exp(l * e.inv_tau - lt[r]);
          d = e.a1 * d + e.a2 * dt;
        }
        acc[i][j][r] = d;
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
      for (int k = run0 + lane; k < run1; k += 64) {
        const uint32_t w = e.ent[k];
        region[staged_at(w & 15, (int)(w >> 4) - e.v0 - col0)] -= e.a2 * e.ent_p[k];
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
      if (row < rows_left && col0 + vcol < e.ldd) {
        uint16_t* out = e.dl + (int64_t)(row0 + row) * e.ldd + col0 + vcol;
        if constexpr (TERMS == 1) {
          *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        } else {
          float x[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int t = 0; t < TERMS; ++t) {
            uint32_t b[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) b[k] = bf16_term(x[k]);
            *reinterpret_cast<uint2*>(out + t * e.plane) = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
          }
        }
      }
    }
    __builtin_amdgcn_s_waitcnt(kWaitLgkm);   // the slice has been read
  }
  if (e.col_sums) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      cs[k] += __shfl_xor(cs[k], 16, 64);
      cs[k] += __shfl_xor(cs[k], 32, 64);
    }
    if (q == 0 && rows_left > 0) {
      float* out = e.col_sums + (int64_t)(row0 / 128) * e.ld_sums + col0 + vcol;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (col0 + vcol + k < ncols) out[k] = cs[k];
    }
  }
}

}  // namespace asx
