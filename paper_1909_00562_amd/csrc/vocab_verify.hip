// Verification of drafted words against the target's probabilities (speculative sampling): entry points and kernels.
//
// A word is told from its neighbour by where a random number falls among sums over the vocabulary, so that probabilities are computed
// in 64 bits: with 128000 borders, each off by 1e-8 as in fp32, one draw in a thousand would go to another word.  fp64 additions and
// multiplications run at fp32's rate here.
// Two launches.  The first one reads all rows once, a chunk of a row per block: its maximum and the sum of exp relative to it.  In
// the second every block of a sequence joins those, finds how many words are accepted, and adds up the weights max(p - q, 0) of its
// chunk; the sequence's last block to arrive finds the chunk in which u times the sum lies, and in it the word.
#include "../../include/vocab_ops.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "common.h"
#include "status.h"

namespace asx {
namespace {

typedef uint32_t vu32x4_t __attribute__((ext_vector_type(4)));

constexpr int kVThreads = 256, kVPer = 32, kVChunk = kVThreads * kVPer;   // logits of a thread and of a block
constexpr int kVerifyMaxT = 64;

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
  double2* sums;       // [B][chunks]: of max(p - q, 0), of p
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
template <typename TE> __global__ __launch_bounds__(kVThreads) void verify_stats_kernel(VerifyDev a) {
  constexpr int W = 16 / sizeof(TE);
  __shared__ float s_m[4];
  __shared__ double s_sum[4];
  const int rows = 2 * a.T + 1, b = blockIdx.y / rows, j = blockIdx.y - b * rows;
  const int tid = threadIdx.x, wave = tid >> 6;
  if (j == 0 && blockIdx.x == 0 && tid == 0) a.ticket[b] = 0;
  // the target's row t is looked at behind t words, the draft's with its word
  const int t = j <= a.T ? j : j - a.T - 1, ahead = j <= a.T ? t : t + 1;
  for (int i = 0; i < ahead; ++i)
    if (!is_word(a.drafted[(int64_t)b * a.T + i], a.V)) return;
  const TE* row = j <= a.T ? reinterpret_cast<const TE*>(a.target) + ((int64_t)b * (a.T + 1) + t) * a.ld_target
                           : reinterpret_cast<const TE*>(a.draft) + ((int64_t)b * a.T + t) * a.ld_draft;
  float l[kVPer];
#pragma unroll
  for (int i = 0; i < kVPer / W; ++i) {
    const int v0 = blockIdx.x * kVChunk + (i * kVThreads + tid) * W;
    ld_logits<TE>(row, v0 < a.V ? v0 : a.V, a.V, l + i * W);
  }
  float m = -INFINITY;
  int bad = 0;
#pragma unroll
  for (int i = 0; i < kVPer; ++i) {
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
    const double m64 = m;
#pragma unroll
    for (int i = 0; i < kVPer; ++i) sum += exp2_64(((double)l[i] - m64) * a.c);
  }
  sum = wave_sum64(sum);
  if ((tid & 63) == 0) s_sum[wave] = sum;
  __syncthreads();
  if (tid == 0) a.part[(int64_t)blockIdx.y * a.chunks + blockIdx.x] = {(s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]), m, bad};
}

// ---- the words ---------------------------------------------------------------------
struct RowStat {
  double m, inv_z;   // p[v] = 2^((l[v] - m) c) inv_z
};
template <typename TE> struct Weights {
  const TE *p_row, *q_row;   // q_row: null where p alone counts
  RowStat p, q;
  double c;
  __device__ __forceinline__ void at(float lp, float lq, bool rest, double& r, double& pv) const {
    pv = exp2_64(((double)lp - p.m) * c) * p.inv_z;
    r = pv;
    if (rest) r = fmax(pv - exp2_64(((double)lq - q.m) * c) * q.inv_z, 0.0);
  }
};

template <typename TE> __global__ __launch_bounds__(kVThreads) void verify_words_kernel(VerifyDev a) {
  constexpr int W = 16 / sizeof(TE);
  __shared__ RowStat s_stat[2 * kVerifyMaxT + 1];
  __shared__ int8_t s_bad[2 * kVerifyMaxT + 1], s_ok[kVerifyMaxT], s_word[kVerifyMaxT];
  __shared__ int s_n, s_state, s_last, s_chunk, s_found;
  __shared__ double s_r[4], s_p[4], s_theta;
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, T = a.T, V = a.V;
  const int64_t first = (int64_t)b * T;
  const TE* target = reinterpret_cast<const TE*>(a.target) + (int64_t)b * (T + 1) * a.ld_target;
  const TE* draft = reinterpret_cast<const TE*>(a.draft) + first * a.ld_draft;
  if (tid < T) s_word[tid] = is_word(a.drafted[first + tid], V);
  __syncthreads();
  int words = 0;   // drafted ones
  while (words < T && s_word[words]) ++words;
  // a wave joins the parts of a row
  for (int i = wave; i < 2 * words + 1; i += 4) {
    const int j = i <= words ? i : i - words + T;   // (target rows 0 .. words, draft rows 0 .. words - 1)
    const VerifyPart* part = a.part + ((int64_t)b * (2 * T + 1) + j) * a.chunks;
    float m = -INFINITY;
    int bad = 0;
    for (int k = lane; k < a.chunks; k += 64) {
      m = fmaxf(m, part[k].m);
      bad |= part[k].bad;
    }
    m = wave_max(m);
    bad = __any(bad) || !(m > -INFINITY);
    double z = 0;
    if (!bad)
      for (int k = lane; k < a.chunks; k += 64)
        if (part[k].m > -INFINITY) z += part[k].sum * exp2_64(((double)part[k].m - (double)m) * a.c);
    z = wave_sum64(z);
    if (lane == 0) {
      s_stat[j] = {m, 1.0 / z};
      s_bad[j] = bad;
    }
  }
  __syncthreads();
  if (tid < words) {
    const int32_t x = a.drafted[first + tid];
    const RowStat p = s_stat[tid], q = s_stat[T + 1 + tid];
    const double px = exp2_64(((double)ld_elem<TE>(target + tid * a.ld_target, x) - p.m) * a.c) * p.inv_z;
    const double qx = exp2_64(((double)ld_elem<TE>(draft + tid * a.ld_draft, x) - q.m) * a.c) * q.inv_z;
    s_ok[tid] = s_bad[tid] || s_bad[T + 1 + tid] ? 2 : (double)a.u_accept[first + tid] * qx < px;
  }
  __syncthreads();
  if (tid == 0) {
    int n = 0;
    while (n < words && s_ok[n] == 1) ++n;
    s_n = n;
    s_state = (n < words && s_ok[n] == 2) || s_bad[n] ? 2 : n < words;   // 0: from p, 1: what is left of p, 2: no distribution
  }
  __syncthreads();
  const int n = s_n, state = s_state;
  const bool rest = state == 1;
  if (blockIdx.x == 0) {
    if (tid == 0) a.n_accepted[b] = n;
    if (tid <= T && (tid != n || state == 2)) a.words[first + b + tid] = tid < n ? a.drafted[first + tid] : -1;
  }
  if (state == 2) return;
  Weights<TE> w;
  w.p_row = target + n * a.ld_target;
  w.q_row = rest ? draft + n * a.ld_draft : w.p_row;
  w.p = s_stat[n];
  w.q = s_stat[rest ? T + 1 + n : n];
  w.c = a.c;
  // this chunk's weights
  double r = 0, p = 0;
#pragma unroll 2
  for (int i = 0; i < kVPer / W; ++i) {
    const int v0 = blockIdx.x * kVChunk + (i * kVThreads + tid) * W;
    if (v0 >= V) break;
    float lp[W], lq[W];
    ld_logits<TE>(w.p_row, v0, V, lp);
    if (rest) ld_logits<TE>(w.q_row, v0, V, lq);
#pragma unroll
    for (int e = 0; e < W; ++e) {
      double rv, pv;
      w.at(lp[e], rest ? lq[e] : 0.f, rest, rv, pv);
      r += rv;
      p += pv;
    }
  }
  r = wave_sum64(r);
  p = wave_sum64(p);
  if (lane == 0) {
    s_r[wave] = r;
    s_p[wave] = p;
  }
  __syncthreads();
  double2* sums = a.sums + (int64_t)b * a.chunks;
  if (tid == 0) {
    __hip_atomic_store(&sums[blockIdx.x].x, (s_r[0] + s_r[1]) + (s_r[2] + s_r[3]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(&sums[blockIdx.x].y, (s_p[0] + s_p[1]) + (s_p[2] + s_p[3]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __threadfence();
    s_last = __hip_atomic_fetch_add(&a.ticket[b], 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.chunks - 1;
  }
  __syncthreads();
  if (!s_last) return;
  // the sequence's last block: the chunk, added up in order whichever block this is
  if (tid == 0) {
    auto sum_of = [&](int k, bool of_p) {
      return __hip_atomic_load(of_p ? &sums[k].y : &sums[k].x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    double all = 0;
    for (int k = 0; k < a.chunks; ++k) all += sum_of(k, false);
    const bool of_p = !(all > 0);   // nothing is left: p
    if (of_p) {
      all = 0;
      for (int k = 0; k < a.chunks; ++k) all += sum_of(k, true);
    }
    const double theta = fmax((double)a.u_next[b], 0.0) * all;
    double ahead = 0;
    int chunk = -1, some = 0;
    double left = INFINITY;
    for (int k = 0; k < a.chunks && chunk < 0; ++k) {
      const double s = sum_of(k, of_p);
      if (s > 0) some = k;
      if (ahead + s > theta) {
        chunk = k;
        left = theta - ahead;
      }
      ahead += s;
    }
    s_chunk = chunk < 0 ? some : chunk;
    s_theta = left;
    s_state = of_p;
    s_found = 1 << 30;
    s_n = -1;
  }
  __syncthreads();
  const bool of_p = s_state;
  const int v1 = s_chunk * kVChunk + tid * kVPer;   // consecutive logits per thread: running sums go by the words' order
  double own = 0;
  float lp[kVPer], lq[kVPer];
#pragma unroll
  for (int i = 0; i < kVPer / W; ++i) {
    const int v0 = v1 + i * W;
    ld_logits<TE>(w.p_row, v0 < V ? v0 : V, V, lp + i * W);
    ld_logits<TE>(w.q_row, v0 < V ? v0 : V, V, lq + i * W);
  }
  const bool subtract = rest && !of_p;
#pragma unroll 4
  for (int i = 0; i < kVPer; ++i) {
    double rv, pv;
    w.at(lp[i], lq[i], subtract, rv, pv);
    own += rv;
  }
  double run = own;   // inclusive over the block
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double x = __shfl_up(run, o, 64);
    if (lane >= o) run += x;
  }
  if (lane == 63) s_r[wave] = run;
  __syncthreads();
  for (int i = 0; i < wave; ++i) run += s_r[i];
  if (run > s_theta) atomicMin(&s_found, tid);
  if (own > 0) atomicMax(&s_n, tid);
  __syncthreads();
  const bool none = s_found == 1 << 30;      // (rounding, or u >= 1: the last word of a weight above 0)
  if (tid != (none ? s_n : s_found)) return;
  double at = run - own;
  int word = -1;
  for (int i = 0; i < kVPer; ++i) {
    double rv, pv;
    w.at(lp[i], lq[i], subtract, rv, pv);
    at += rv;
    if (rv > 0) word = v1 + i;
    if (!none && at > s_theta && rv > 0) break;
  }
  a.words[first + b + n] = word;
}

struct VerifyLayout {
  int chunks;
  size_t part, sums, ticket, total;
};
VerifyLayout verify_layout(const vo_verify* s) {
  VerifyLayout L;
  L.chunks = (s->V + kVChunk - 1) / kVChunk;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  L.part = 0;
  L.sums = up((size_t)s->B * (2 * s->T + 1) * L.chunks * sizeof(VerifyPart));
  L.ticket = L.sums + up((size_t)s->B * L.chunks * sizeof(double2));
  L.total = L.ticket + up((size_t)s->B * 4);
  return L;
}
bool verify_ok(const vo_verify* s) {
  return s->B >= 1 && s->B <= (1 << 16) && s->T >= 1 && s->T <= kVerifyMaxT && s->V >= 1 && s->V <= (1 << 20) &&
         s->temperature >= 0x1p-10f && s->temperature <= 0x1p10f;
}
bool verify_types(const vo_verify* s) { return s->dtype == AS_F32 || s->dtype == AS_BF16; }
bool al16r(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename TE> hipError_t launch_verify(const VerifyDev& d, hipStream_t st) {
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
    hipLaunchKernelGGL(verify_stats_kernel<TE>, dim3(d.chunks, p.B * rows), dim3(kVThreads), 0, st, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_words_kernel<TE>, dim3(d.chunks, p.B), dim3(kVThreads), 0, st, p);
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
  d.sums = reinterpret_cast<double2*>(ws + L.sums);
  d.ticket = reinterpret_cast<uint32_t*>(ws + L.ticket);
  d.B = shape->B;
  d.T = shape->T;
  d.V = shape->V;
  d.chunks = L.chunks;
  d.c = 1.4426950408889634 / (double)shape->temperature;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const hipError_t err = e == 4 ? launch_verify<float>(d, st) : launch_verify<uint16_t>(d, st);
  return err == hipSuccess ? AS_OK : set_error(AS_ERR_HIP, "vocab_verify: %s", hipGetErrorString(err));
}
