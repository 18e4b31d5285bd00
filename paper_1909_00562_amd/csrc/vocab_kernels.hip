// Kernels around the products of the vocabulary operators: the rows of words, the teacher's lists, the join of the tiles'
// statistics, and what takes gradients to where the caller wants them.
#include <climits>

#include "common.h"
#include "lds_limit.h"
#include "row_threads.h"
#include "vocab.h"
#include "vocab_epi_dev.h"

namespace asx {
namespace {

__device__ __forceinline__ int row_count(const int32_t* n_act, int N) {
  const int v = *n_act;
  return v < 0 ? 0 : (v < N ? v : N);
}

// ---- rows of words --------------------------------------------------------------------
// 16 positions per block.  A block counts the words ahead of its own by reading all targets there (64 KiB at 16384 positions,
// from the L2): a list made ahead by one block would be a launch of its own that everything waits for.  Behind kRowsDirect positions,
// where that reading would grow with their square, a launch counts the words of every kRowsChunk ahead (us, direct / counted: 65536
// positions 33.7 / 21.8, 131072 101 / 34.5; a launch is 5).
constexpr int kRowsBlock = 16;
__device__ __forceinline__ bool is_word(int y, int V, int pad_id) { return y >= 0 && y < V && y != pad_id; }
// words among positions [beg, end), beg % 4 == 0; the sum over the block's 256 threads
__device__ __forceinline__ int count_words(const VocabRows& p, int beg, int end, int* part) {
  const int tid = threadIdx.x;
  int n = 0;
  for (int i0 = beg; i0 < end; i0 += 8192) {   // eight loads together
    int4 y[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u * 1024 + tid * 4;
      y[u] = make_int4(-1, -1, -1, -1);
      if (i + 4 <= end) {
        y[u] = *reinterpret_cast<const int4*>(p.targets + i);
      } else if (i < end) {
        y[u].x = p.targets[i];
        if (i + 1 < end) y[u].y = p.targets[i + 1];
        if (i + 2 < end) y[u].z = p.targets[i + 2];
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      n += is_word(y[u].x, p.V, p.pad_id) + is_word(y[u].y, p.V, p.pad_id) + is_word(y[u].z, p.V, p.pad_id) + is_word(y[u].w, p.V, p.pad_id);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((tid & 63) == 0) part[tid >> 6] = n;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}
__global__ __launch_bounds__(256) void vocab_count_kernel(VocabRows p) {
  __shared__ int part[4];
  const int64_t beg = (int64_t)blockIdx.x * kRowsChunk;
  const int n = count_words(p, (int)beg, beg + kRowsChunk < p.N ? (int)(beg + kRowsChunk) : p.N, part);
  if (threadIdx.x == 0) p.chunk_words[blockIdx.x] = n;
}
__global__ __launch_bounds__(256) void vocab_rows_kernel(VocabRows p) {
  __shared__ int part[4], chunk_part[4], place[kRowsBlock];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n0 = blockIdx.x * kRowsBlock;
  const int chunks = p.chunk_words ? n0 / kRowsChunk : 0;
  int ahead = 0;   // in whole chunks
  if (chunks > 0) {
    for (int i = tid; i < chunks; i += 256) ahead += p.chunk_words[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) ahead += __shfl_xor(ahead, o, 64);
    if (lane == 0) chunk_part[wave] = ahead;
    __syncthreads();
    ahead = chunk_part[0] + chunk_part[1] + chunk_part[2] + chunk_part[3];
  }
  const int before = ahead + count_words(p, chunks * kRowsChunk, n0, part);
  if (wave == 0) {
    const int n = n0 + lane;
    const bool in = lane < kRowsBlock && n < p.N;
    const int y = in ? p.targets[n] : -1;
    const bool word = in && is_word(y, p.V, p.pad_id);
    const uint64_t m = __ballot(word);
    const int r = before + __popcll(m & ((1ull << lane) - 1));
    if (lane < kRowsBlock) place[lane] = word ? r : -1;
    if (in) {
      p.row_pos[n] = word ? r : -1;
      if (word) {
        p.rows[r] = n;
        p.y[r] = y;
      } else {
        if (p.tok_loss) p.tok_loss[n] = 0.f;
        if (p.tok_distill) p.tok_distill[n] = 0.f;
        if (p.argmax) p.argmax[n] = p.pad_id;
      }
    }
    if (lane == 0 && n0 + kRowsBlock >= p.N) *p.n_act = before + __popcll(m);
    if (lane == 0 && blockIdx.x == 0) *p.ticket = 0;
  }
  __syncthreads();
  // the rows themselves, a wave each, its four rows' loads together
  if (!p.f32) {   // H % 8 == 0
    for (int c = lane * 8; c < p.H; c += 512) {
      uint4 x[kRowsBlock / 4];
#pragma unroll
      for (int k = 0; k < kRowsBlock / 4; ++k) {
        const int j = wave + 4 * k;
        x[k] = place[j] < 0 ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.h) + (int64_t)(n0 + j) * p.H + c);
      }
#pragma unroll
      for (int k = 0; k < kRowsBlock / 4; ++k) {
        const int r = place[wave + 4 * k];
        if (r >= 0) *reinterpret_cast<uint4*>(p.hc + (int64_t)r * p.ldH + c) = x[k];
      }
    }
  } else {
    const bool vec = p.H % 4 == 0;
    for (int c = lane * 4; c < p.ldH; c += 256) {
      float x[kRowsBlock / 4][4];
#pragma unroll
      for (int k = 0; k < kRowsBlock / 4; ++k) {
        const int j = wave + 4 * k;
        const float* src = reinterpret_cast<const float*>(p.h) + (int64_t)(n0 + j) * p.H + c;
        const bool in = place[j] >= 0;
        if (vec && c < p.H) {
          const f32x4_t v = in ? *reinterpret_cast<const f32x4_t*>(src) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 4; ++e) x[k][e] = v[e];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[k][e] = in && c + e < p.H ? src[e] : 0.f;
        }
      }
#pragma unroll
      for (int k = 0; k < kRowsBlock / 4; ++k) {
        const int r = place[wave + 4 * k];
        if (r < 0) continue;
#pragma unroll
        for (int t = 0; t < 3; ++t) {
          uint32_t b[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) b[e] = bf16_term(x[k][e]);
          *reinterpret_cast<uint2*>(p.hc + t * p.plane + (int64_t)r * p.ldH + c) = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
        }
      }
    }
  }
}

// ---- fp32 operands as terms -------------------------------------------------------------
// Four columns per thread; bound by memory (4 bytes in, 6 out).
__global__ __launch_bounds__(256) void vocab_terms_kernel(const float* __restrict__ src, int rows, int H, uint16_t* __restrict__ dst,
                                                          int64_t ldH, int64_t plane, int quads_log) {
  const int64_t r = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> quads_log;
  if (r >= rows) return;
  const int lane = threadIdx.x & ((1 << quads_log) - 1);
  const float* x0 = src + r * H;
  for (int c = lane * 4; c < ldH; c += 4 << quads_log) {
    float x[4];
    if (H % 4 == 0 && c + 4 <= H) {
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(x0 + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = c + e < H ? x0[c + e] : 0.f;
    }
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      uint32_t b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = bf16_term(x[e]);
      *reinterpret_cast<uint2*>(dst + t * plane + r * ldH + c) = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
    }
  }
}

// ---- the teacher's lists ------------------------------------------------------------------
// A block per group of 16 rows, a wave per row.  Softmax over the row's entries; entries with the same id become one with all
// of their probability (the first of them); a counting sort of the group's entries by strip of 64 columns.  The order inside a
// strip is not fixed and nothing depends on it: no two entries are of the same row and column, and place[] finds a row's entries.
__global__ __launch_bounds__(1024) void vocab_teacher_kernel(VocabTeacher p) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int wsum[16];
  const int R = row_count(p.n_act, p.N), g = blockIdx.x;
  if (g * kVocabGroup >= R) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = p.K, K4 = (K + 3) & ~3, r = g * kVocabGroup + wave;
  int* ids = reinterpret_cast<int*>(smem) + wave * K4;
  float* prob = reinterpret_cast<float*>(smem) + 16 * K4 + wave * K4;
  int* hist = reinterpret_cast<int*>(smem) + 32 * K4;
  for (int i = tid; i < p.strips; i += 1024) hist[i] = 0;
  constexpr int PER = kTeacherMaxK / 64;
  int id[PER];
  float P[PER];
  bool first[PER];
  const bool row = r < R;
  const int64_t at = row ? (int64_t)p.rows[r] * K : 0;
  float z[PER], top = -INFINITY;
  bool any = false, in[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int k = lane + 64 * j;
    id[j] = row && k < K ? p.ids[at + k] : -1;
    z[j] = row && k < K ? p.logits[at + k] : -INFINITY;   // (not used where the id is none)
    in[j] = id[j] >= 0 && id[j] < p.V && z[j] != -INFINITY;
    if (!in[j]) id[j] = -1;
    any = any || in[j];
    top = in[j] ? fmaxf(top, z[j]) : top;
  }
  top = wave_max(top);
  any = __ballot(any) != 0;
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    z[j] = (z[j] - top) * p.inv_tau;
    P[j] = in[j] ? expf(z[j]) : 0.f;
    sum += P[j];
  }
  sum = wave_sum(sum);
  const float log_sum = logf(sum), inv = 1.f / sum;
  float plp = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    P[j] = in[j] ? P[j] * inv : 0.f;
    if (P[j] != 0.f) plp += P[j] * (z[j] - log_sum);   // (NaN stays)
    if (lane + 64 * j < K4) {
      ids[lane + 64 * j] = id[j];
      prob[lane + 64 * j] = P[j];
    }
  }
  plp = wave_sum(plp);
  if (row && lane == 0) {
    p.p_log_p[r] = any ? plp : 0.f;
    p.seen[r] = any ? 1 : 0;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    first[j] = in[j];
    P[j] = 0.f;
  }
  for (int k0 = 0; k0 < K4; k0 += 4) {
    const int4 o4 = *reinterpret_cast<const int4*>(ids + k0);
    const float4 q4 = *reinterpret_cast<const float4*>(prob + k0);
    const int o[4] = {o4.x, o4.y, o4.z, o4.w};
    const float q[4] = {q4.x, q4.y, q4.z, q4.w};
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (64 * j >= K) continue;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool same = in[j] && o[u] == id[j];
        P[j] += same ? q[u] : 0.f;
        first[j] = first[j] && !(same && k0 + u < lane + 64 * j);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (first[j]) atomicAdd(hist + id[j] / kVocabStrip, 1);
  __syncthreads();
  // exclusive prefix of the strips' counts
  const int per = (p.strips + 1023) / 1024, beg = tid * per;
  int mine = 0;
  for (int i = beg; i < beg + per && i < p.strips; ++i) mine += hist[i];
  int pre = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(pre, o, 64);
    if (lane >= o) pre += t;
  }
  if (lane == 63) wsum[wave] = pre;
  __syncthreads();
  int base = g * kVocabGroup * K, total = 0;
  for (int w = 0; w < 16; ++w) {
    if (w < wave) base += wsum[w];
    total += wsum[w];
  }
  int32_t* runs = p.runs + (int64_t)g * (p.strips + 1);
  int here = base + pre - mine;
  for (int i = beg; i < beg + per && i < p.strips; ++i) {
    const int c = hist[i];
    runs[i] = here;
    hist[i] = here;
    here += c;
  }
  if (tid == 0) runs[p.strips] = g * kVocabGroup * K + total;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int k = lane + 64 * j;
    int to = -1;
    if (first[j]) {
      to = atomicAdd(hist + id[j] / kVocabStrip, 1);
      p.ent[to] = (uint32_t)id[j] << 4 | (uint32_t)wave;
      p.ent_p[to] = P[j];
    }
    if (row && k < K) p.place[(int64_t)r * K + k] = to;
  }
}

// ---- joining the statistics ------------------------------------------------------------------
struct Stat {
  float m, s, t;
  int idx;
};
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b, float inv_tau) {
  constexpr float L2E = 1.4426950408889634f;
  Stat r;
  r.m = fmaxf(a.m, b.m);
  const float da = a.m == r.m ? 0.f : (a.m - r.m) * L2E, db = b.m == r.m ? 0.f : (b.m - r.m) * L2E;
  r.s = a.s * __builtin_amdgcn_exp2f(da) + b.s * __builtin_amdgcn_exp2f(db);
  r.t = a.t * __builtin_amdgcn_exp2f(da * inv_tau) + b.t * __builtin_amdgcn_exp2f(db * inv_tau);
  r.idx = a.m > b.m ? a.idx : (b.m > a.m ? b.idx : (a.idx < b.idx ? a.idx : b.idx));
  return r;
}

// RPB rows per block, 1024 / RPB threads per row that take every (1024 / RPB)-th part, eight at a time: their loads together, one
// maximum, and sums against it; losses of the rows, and by the block that is through last their sums in double, in a fixed order.
template <int RPB, bool TEACH, bool ARG>
__global__ __launch_bounds__(1024) void vocab_finish_kernel(VocabFinish p) {
  constexpr int PH = 1024 / RPB, U = 8;
  constexpr float L2E = 1.4426950408889634f;
  __shared__ Stat part[16 * RPB];
  __shared__ float sh_tau[RPB];
  __shared__ double sd[2][16];
  __shared__ int last_block;
  const int R = row_count(p.n_act, p.N), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row0 = blockIdx.x * RPB, r = row0 + tid % RPB, phase = tid / RPB;
  if (row0 < R) {
    // A wave per row of the teacher's entries: their probabilities' sum and that of p l / tau, ahead of what log q needs besides
    constexpr int RW = RPB / 16;
    float pl[RW] = {}, ps[RW] = {};
    bool has[RW] = {};   // an entry
    if (TEACH && p.last) {
#pragma unroll
      for (int j = 0; j < RW; ++j) {
        const int row = row0 + wave + 16 * j;
        if (row >= R) continue;
        has[j] = p.seen[row] != 0;
        for (int k = lane; k < p.K; k += 64) {
          const int at = p.place[(int64_t)row * p.K + k];
          if (at < 0) continue;
          const float q = p.ent_p[at];
          if (q != 0.f) {
            pl[j] += q * (p.ent_l[at] * p.inv_tau);
            ps[j] += q;
          }
        }
      }
    }
    Stat st{-INFINITY, 0.f, 0.f, INT_MAX};
    if (r < R) {
      for (int i0 = phase; i0 < p.parts; i0 += U * PH) {
        float2 ms[U];
        float t[U];
        int idx[U];
        Stat g{-INFINITY, 0.f, 0.f, INT_MAX};
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + u * PH;
          const int64_t at = (int64_t)(i < p.parts ? i : i0) * p.ldr + r;
          ms[u] = p.stat[at];
          t[u] = TEACH ? p.stat_tau[at] : 0.f;
          idx[u] = ARG ? p.stat_idx[at] : INT_MAX;
          if (i >= p.parts) {
            ms[u] = make_float2(-INFINITY, 0.f);
            t[u] = 0.f;
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) g.m = fmaxf(g.m, ms[u].x);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float d = ms[u].x == g.m ? 0.f : (ms[u].x - g.m) * L2E;
          g.s += ms[u].y * __builtin_amdgcn_exp2f(d);
          if constexpr (TEACH) g.t += t[u] * __builtin_amdgcn_exp2f(d * p.inv_tau);
          if constexpr (ARG) g.idx = ms[u].x == g.m && idx[u] < g.idx ? idx[u] : g.idx;
        }
        st = join(st, g, p.inv_tau);
      }
    }
    // what the row's thread needs besides, on its way meanwhile
    const bool mine = tid < RPB && r < R;
    const float at_word = mine && p.last ? p.at_word[r] : 0.f;
    const int n = mine && p.last ? p.rows[r] : 0;
    const bool seen = TEACH && mine && p.last ? p.seen[r] != 0 : false;
    // a wave's threads of the row, then the waves'
#pragma unroll
    for (int o = RPB; o < 64; o <<= 1) {
      Stat other;
      other.m = __shfl_xor(st.m, o, 64);
      other.s = __shfl_xor(st.s, o, 64);
      other.t = TEACH ? __shfl_xor(st.t, o, 64) : 0.f;
      other.idx = ARG ? __shfl_xor(st.idx, o, 64) : INT_MAX;
      st = join(st, other, p.inv_tau);
    }
    if (lane < RPB) part[wave * RPB + lane] = st;
    __syncthreads();
    if (mine) {
      Stat w[16];
      st = Stat{-INFINITY, 0.f, 0.f, INT_MAX};
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        w[k] = part[k * RPB + tid];
        st.m = fmaxf(st.m, w[k].m);
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float d = w[k].m == st.m ? 0.f : (w[k].m - st.m) * L2E;
        st.s += w[k].s * __builtin_amdgcn_exp2f(d);
        if constexpr (TEACH) st.t += w[k].t * __builtin_amdgcn_exp2f(d * p.inv_tau);
        if constexpr (ARG) st.idx = w[k].m == st.m && w[k].idx < st.idx ? w[k].idx : st.idx;
      }
      if (!p.first) {
        const float4 q = p.run[r];
        st = join(Stat{q.x, q.y, q.z, __builtin_bit_cast(int, q.w)}, st, p.inv_tau);
      }
      if (!p.last) {
        p.run[r] = make_float4(st.m, st.s, st.t, __builtin_bit_cast(float, st.idx));
      } else {
        const float lse = st.m + logf(st.s), loss = lse - at_word;
        p.lse[r] = lse;
        __hip_atomic_store(p.loss_ws + r, loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (p.tok_loss) p.tok_loss[n] = loss;
        if (p.argmax) p.argmax[n] = st.idx == INT_MAX ? 0 : st.idx;
        if constexpr (TEACH) {
          const float lt = seen ? st.m * p.inv_tau + logf(st.t) : INFINITY;
          p.lse_tau[r] = lt;
          sh_tau[tid] = lt;
        }
      }
    }
    if (TEACH && p.last) {
#pragma unroll
      for (int j = 0; j < RW; ++j) {
        pl[j] = wave_sum(pl[j]);
        ps[j] = wave_sum(ps[j]);
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < RW; ++j) {
        const int row = row0 + wave + 16 * j;
        if (row >= R || lane != 0) continue;
        const float lt = sh_tau[wave + 16 * j], d = has[j] ? p.tau2 * (p.p_log_p[row] - (pl[j] - ps[j] * lt)) : 0.f;   // (NaN stays)
        __hip_atomic_store(p.distill_ws + row, d, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (p.tok_distill) p.tok_distill[p.rows[row]] = d;
      }
    }
  }
  const int blocks = R > 0 ? (R + RPB - 1) / RPB : 1;   // with rows; the others are done
  if (!p.last || (int)blockIdx.x >= blocks) return;
  if (blocks > 1) {
    __builtin_amdgcn_s_waitcnt(0);   // the wave's losses are where every XCD sees them (stored past the caches)
    __syncthreads();
    if (tid == 0) last_block = __hip_atomic_fetch_add(p.ticket, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == blocks - 1;
    __syncthreads();
    if (!last_block) return;
  } else {
    __syncthreads();
  }
  double a = 0.0, b = 0.0;
  for (int i0 = tid; i0 < R; i0 += 8192) {   // eight loads together
    float x[8], y[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u * 1024 < R ? i0 + u * 1024 : i0;
      x[u] = __hip_atomic_load(p.loss_ws + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      y[u] = TEACH ? __hip_atomic_load(p.distill_ws + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (i0 + u * 1024 < R) {
        a += (double)x[u];
        b += (double)y[u];
      }
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    a += __shfl_xor(a, o, 64);
    b += __shfl_xor(b, o, 64);
  }
  if (lane == 0) {
    sd[0][wave] = a;
    sd[1][wave] = b;
  }
  __syncthreads();
  if (tid == 0) {
    a = b = 0.0;
    for (int w = 0; w < 16; ++w) {
      a += sd[0][w];
      b += sd[1][w];
    }
    *p.loss_sum = (float)a;
    *p.n_tok = R;
    if constexpr (TEACH) *p.distill_sum = (float)b;
  }
}

// ---- gradients on their way out ------------------------------------------------------------------
// 2^tpr_log threads per row of dh; further blocks for db: 64 words each, four phases of every fourth part of the rows, eight loads
// together, the phases in order
template <typename TE, int VEC>
__global__ __launch_bounds__(256) void vocab_out_grads_kernel(VocabOutGrads p, int tpr_log, int row_blocks) {
  if ((int)blockIdx.x >= row_blocks) {
    __shared__ float red[4][64];
    const int c = threadIdx.x & 63, phase = threadIdx.x >> 6, v = ((int)blockIdx.x - row_blocks) * 64 + c;
    const int parts = (row_count(p.n_act, p.N) + p.sum_rows - 1) / p.sum_rows;
    float s = 0.f;
    if (v < p.V) {
#pragma unroll 8
      for (int i = phase; i < parts; i += 4) s += p.sums[(int64_t)i * p.ld_sums + v];
    }
    red[phase][c] = s;
    __syncthreads();
    if (phase == 0 && v < p.V) st_elem<TE>(reinterpret_cast<TE*>(p.db), v, p.alpha * (((red[0][c] + red[1][c]) + red[2][c]) + red[3][c]));
    return;
  }
  const int64_t n = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> tpr_log;
  if (n >= p.N) return;
  const int lane = threadIdx.x & ((1 << tpr_log) - 1), at = p.row_pos[n], r = at < p.N ? at : -1, H = p.H;
  const float* from = p.src + (int64_t)(r < 0 ? 0 : r) * p.ld;
  TE* out = reinterpret_cast<TE*>(p.dh) + n * H;
  for (int c = lane * VEC; c < H; c += VEC << tpr_log) {
    if constexpr (VEC == 1) {
      st_elem<TE>(out, c, r < 0 ? 0.f : p.alpha * from[c]);
    } else {
      f32x4_t v = {0.f, 0.f, 0.f, 0.f};
      if (r >= 0) v = *reinterpret_cast<const f32x4_t*>(from + c) * p.alpha;
      if constexpr (sizeof(TE) == 2) *reinterpret_cast<uint2*>(out + c) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
      else *reinterpret_cast<f32x4_t*>(out + c) = v;
    }
  }
}

}  // namespace

hipError_t launch_vocab_rows(const VocabRows& p, hipStream_t st) {
  if (p.chunk_words) {
    hipLaunchKernelGGL(vocab_count_kernel, dim3((p.N + kRowsChunk - 1) / kRowsChunk), dim3(256), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(vocab_rows_kernel, dim3((p.N + kRowsBlock - 1) / kRowsBlock), dim3(256), 0, st, p);
  return hipGetLastError();
}

hipError_t launch_vocab_terms(const float* src, int rows, int H, uint16_t* dst, int64_t ldH, int64_t plane, hipStream_t st) {
  const int log = row_threads_log(rows, ldH / 4);
  const int64_t blocks = (((int64_t)rows << log) + 255) / 256;
  hipLaunchKernelGGL(vocab_terms_kernel, dim3((unsigned)blocks), dim3(256), 0, st, src, rows, H, dst, ldH, plane, log);
  return hipGetLastError();
}

hipError_t launch_vocab_teacher(const VocabTeacher& p, hipStream_t st) {
  const int smem = (32 * ((p.K + 3) / 4 * 4) + p.strips) * 4;
  static LdsLimit limit;
  const hipError_t e = limit.raise(reinterpret_cast<const void*>(vocab_teacher_kernel), 128 * 1024);
  if (e != hipSuccess) return e;
  if (smem > 128 * 1024) return hipErrorInvalidValue;
  hipLaunchKernelGGL(vocab_teacher_kernel, dim3((p.N + kVocabGroup - 1) / kVocabGroup), dim3(1024), smem, st, p);
  return hipGetLastError();
}

hipError_t launch_vocab_finish(const VocabFinish& p, hipStream_t st) {
  // Few rows: more threads per row, since a row's parts are read one after the other.
#define ASX_FINISH(RPB, TEACH, ARG) \
  hipLaunchKernelGGL((vocab_finish_kernel<RPB, TEACH, ARG>), dim3((p.N + RPB - 1) / RPB), dim3(1024), 0, st, p)
#define ASX_FINISH_OF(TEACH, ARG)               \
  do {                                          \
    if (p.N <= 1024) ASX_FINISH(16, TEACH, ARG); \
    else ASX_FINISH(32, TEACH, ARG);            \
  } while (0)
  if (p.stat_tau) ASX_FINISH_OF(true, false);
  else if (p.stat_idx) ASX_FINISH_OF(false, true);
  else ASX_FINISH_OF(false, false);
#undef ASX_FINISH_OF
#undef ASX_FINISH
  return hipGetLastError();
}

hipError_t launch_vocab_out_grads(const VocabOutGrads& p, bool bf16, hipStream_t st) {
  const bool vec = p.H % 4 == 0;   // (bf16 rows: H % 8 == 0)
  const int log = row_threads_log(p.N, vec ? p.H / 4 : p.H);
  const int row_blocks = (int)((((int64_t)p.N << log) + 255) / 256), blocks = row_blocks + (p.db ? (p.V + 63) / 64 : 0);
  if (bf16) hipLaunchKernelGGL((vocab_out_grads_kernel<uint16_t, 4>), dim3(blocks), dim3(256), 0, st, p, log, row_blocks);
  else if (vec) hipLaunchKernelGGL((vocab_out_grads_kernel<float, 4>), dim3(blocks), dim3(256), 0, st, p, log, row_blocks);
  else hipLaunchKernelGGL((vocab_out_grads_kernel<float, 1>), dim3(blocks), dim3(256), 0, st, p, log, row_blocks);
  return hipGetLastError();
}

}  // namespace asx
