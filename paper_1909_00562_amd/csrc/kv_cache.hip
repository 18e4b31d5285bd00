// Paged cache of keys and values: rows into it and out of it, as they are or in 8 bits (entry points and kernels).
//
// A row is a token's D values of one head, of keys or of values; the largest magnitude of its values, which the scale of its codes is made
// of, is found by the lanes that hold it.  Bound by memory: each value is read once and each code written once.
#include "kv_cache.h"

#include <type_traits>

#include "common.h"
#include "status.h"

namespace asx {

as_status kv_check_cache(const kc_cache* c) {
  if (!c) return set_error(AS_ERR_NULL, "cache is NULL");
  if ((c->dtype != AS_F32 && c->dtype != AS_BF16) || (c->cache_type != c->dtype && !kv_coded(c->cache_type)))
    return set_error(AS_ERR_DTYPE, "cache of type %d for values of dtype %d", c->cache_type, c->dtype);
  if (c->pages < 1 || c->page < kKvTile || c->page > 4096 || c->page % kKvTile != 0 || (int64_t)c->pages * c->page >= (int64_t)1 << 31)
    return set_error(AS_ERR_SHAPE, "%d pages of %d tokens", c->pages, c->page);
  if (c->heads < 1 || c->heads > 1024 || c->D < 16 || c->D > 256 || c->D % 16 != 0)
    return set_error(AS_ERR_SHAPE, "%d heads of %d", c->heads, c->D);
  if (c->B < 1 || c->B > (1 << 16) || c->max_pages < 1 || (int64_t)c->B * c->max_pages >= (int64_t)1 << 31 ||
      (int64_t)c->max_pages * c->page >= (int64_t)1 << 31)
    return set_error(AS_ERR_SHAPE, "table of %d sequences, %d pages each of %d tokens", c->B, c->max_pages, c->page);
  return AS_OK;
}

as_status kv_check_pool(const kc_cache* c, const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                        const int32_t* page_table, const char* what) {
  if (!k_pages || !v_pages || !page_table) return set_error(AS_ERR_NULL, "%s: a required pointer is NULL", what);
  if (kv_coded(c->cache_type) ? !k_scales || !v_scales : k_scales || v_scales)
    return set_error(AS_ERR_NULL, "%s: scales belong to caches in 8 bits, and to those alone", what);
  for (const void* p : {k_pages, v_pages, (const void*)k_scales, (const void*)v_scales, (const void*)page_table})
    if (!kv_al16(p)) return set_error(AS_ERR_ALIGN, "%s: a pointer is not 16-byte aligned", what);
  return AS_OK;
}

namespace {

typedef uint32_t ku32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t ku32x2_t __attribute__((ext_vector_type(2)));

struct KvMove {
  const int32_t *seq, *pos, *table;
  int32_t N, heads, D, page, pages, B, max_pages;
  int32_t lanes_log;    // 2^lanes_log lanes to a row, 8 values each
  const void* src[2];   // dense side, keys and values, rows of a token ld apart
  int64_t ld[2];
  void* dst[2];
  void* pool[2];
  float* scales[2];
};

// a token's row of its head 0 in the pool, or -1
__device__ __forceinline__ int64_t row_of(const KvMove& a, int32_t b, int32_t p) {
  if (b < 0 || b >= a.B || p < 0) return -1;
  const int32_t col = (int32_t)((uint32_t)p / (uint32_t)a.page);
  if (col >= a.max_pages) return -1;
  const int32_t id = a.table[(int64_t)b * a.max_pages + col];
  if (id < 0 || id >= a.pages) return -1;
  return (int64_t)id * a.heads * a.page + (p - col * a.page);
}

// PAST: past the caches
template <bool PAST = false> __device__ __forceinline__ void ld8(const uint16_t* p, float (&x)[8]) {
  const ku32x4_t* from = reinterpret_cast<const ku32x4_t*>(p);
  const ku32x4_t q = PAST ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = q[i];
    x[2 * i] = lo_bf16(w);
    x[2 * i + 1] = hi_bf16(w);
  }
}
template <bool PAST = false> __device__ __forceinline__ void ld8(const float* p, float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x4_t* from = reinterpret_cast<const f32x4_t*>(p + 4 * h);
    const f32x4_t q = PAST ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[4 * h + i] = q[i];
  }
}
template <bool PAST, typename V> __device__ __forceinline__ void st_vec(V* p, V v) {
  if constexpr (PAST) __builtin_nontemporal_store(v, p);
  else *p = v;
}
template <bool PAST = false> __device__ __forceinline__ void st8(uint16_t* p, const float (&x)[8]) {
  st_vec<PAST>(reinterpret_cast<ku32x4_t*>(p), ku32x4_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])});
}
template <bool PAST = false> __device__ __forceinline__ void st8(float* p, const float (&x)[8]) {
  st_vec<PAST>(reinterpret_cast<f32x4_t*>(p), f32x4_t{x[0], x[1], x[2], x[3]});
  st_vec<PAST>(reinterpret_cast<f32x4_t*>(p + 4), f32x4_t{x[4], x[5], x[6], x[7]});
}

// eight codes
template <int TYPE> __device__ __forceinline__ ku32x2_t encode8(const float (&x)[8], float inv) {
#pragma clang fp contract(off)   // the product is a float before it is rounded to a code
  ku32x2_t q;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (TYPE == KC_INT8) {
      // of 1.5 2^23 + x the lowest bits are x's, rounded to even
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y = x[4 * h + i] * inv;
        w[i] = __builtin_bit_cast(uint32_t, y + 12582912.f);
      }
      q[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u), __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u);
    } else {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h] * inv, x[4 * h + 1] * inv, 0, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2] * inv, x[4 * h + 3] * inv, w, true);
      q[h] = (uint32_t)w;
    }
  }
  return q;
}
template <int TYPE> __device__ __forceinline__ void decode8(ku32x2_t q, float scale, float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t w = q[h];
    if constexpr (TYPE == KC_INT8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = (float)(int8_t)(w >> (8 * i)) * scale;
    } else {
      const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
      x[4 * h] = a[0] * scale;
      x[4 * h + 1] = a[1] * scale;
      x[4 * h + 2] = b[0] * scale;
      x[4 * h + 3] = b[1] * scale;
    }
  }
}

template <int PATTERN> __device__ __forceinline__ uint32_t max_with(uint32_t x) {
  const uint32_t y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, PATTERN, 0xf, 0xf, true);
  return x > y ? x : y;
}
// over 2^lanes_log neighbouring lanes (the same for all)
__device__ __forceinline__ uint32_t max_of_lanes(uint32_t x, int lanes_log) {
  x = max_with<0xb1>(x);                        // lanes 1 apart
  if (lanes_log > 1) x = max_with<0x4e>(x);     // 2 apart
  if (lanes_log > 2) x = max_with<0x141>(x);    // the other half of 8
  if (lanes_log > 3) x = max_with<0x140>(x);    // the other half of 16
  if (lanes_log > 4) {
    const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = p[0] > p[1] ? p[0] : p[1];
  }
  return x;
}

// A wave moves the same head of keys or of values of ROWS tokens to each of its groups of lanes, neighbours side by side: in the pool their
// rows and their scales follow each other, and the loads of all are on their way together.
template <typename TE, int TYPE, bool WRITE, int ROWS, bool PAST> __global__ __launch_bounds__(256) void kv_move_kernel(KvMove a) {
  constexpr bool kCoded = TYPE == KC_INT8 || TYPE == KC_E4M3;
  const int groups = 64 >> a.lanes_log, lane = threadIdx.x & ((1 << a.lanes_log) - 1), d = lane * 8;
  const int quads = (2 * a.heads + 3) / 4, tile = blockIdx.x / quads, hh = (blockIdx.x - tile * quads) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (hh >= 2 * a.heads) return;
  const int of_v = hh >= a.heads, h = of_v ? hh - a.heads : hh;
  const int n0 = tile * (groups * ROWS) + ((threadIdx.x & 63) >> a.lanes_log);
  const bool here = d < a.D;
  int32_t seq[ROWS], pos[ROWS];
  float x[ROWS][8];
  int64_t row[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int n = n0 + i * groups, at = n < a.N ? n : a.N - 1;
    seq[i] = a.seq[at];
    pos[i] = a.pos[at];
    if (n >= a.N) seq[i] = -1;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
    if constexpr (WRITE)
      if (here) ld8<PAST>(reinterpret_cast<const TE*>(a.src[of_v]) + at * a.ld[of_v] + h * a.D + d, x[i]);
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    row[i] = row_of(a, seq[i], pos[i]);
    if (row[i] >= 0) row[i] += (int64_t)h * a.page;
  }
  if constexpr (WRITE) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if constexpr (!kCoded) {
        if (here && row[i] >= 0) st8(reinterpret_cast<TE*>(a.pool[of_v]) + row[i] * a.D + d, x[i]);
      } else {
        // the largest magnitude, as bits: a NaN's are above infinity's
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t m = __builtin_bit_cast(uint32_t, x[i][e]) & 0x7fffffffu;
          top = m > top ? m : top;
        }
        top = max_of_lanes(top, a.lanes_log);
        constexpr float kPer = TYPE == KC_INT8 ? 1.f / 127.f : 1.f / 448.f;
        const bool finite = top < 0x7f800000u;
        const float scale = fmaxf(__builtin_bit_cast(float, top) * kPer, 0x1p-120f), inv = finite ? 1.f / scale : 0.f;
        if (!finite)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
        if (row[i] >= 0) {
          if (here) *reinterpret_cast<ku32x2_t*>(reinterpret_cast<uint8_t*>(a.pool[of_v]) + row[i] * a.D + d) = encode8<TYPE>(x[i], inv);
          if (lane == 0) a.scales[of_v][row[i]] = finite ? scale : __builtin_nanf("");
        }
      }
    }
  } else {
    ku32x2_t q[ROWS];
    float scale[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      q[i] = ku32x2_t{0u, 0u};
      scale[i] = 0.f;
      if (here && row[i] >= 0) {
        if constexpr (!kCoded) {
          ld8(reinterpret_cast<const TE*>(a.pool[of_v]) + row[i] * a.D + d, x[i]);
        } else {
          q[i] = *reinterpret_cast<const ku32x2_t*>(reinterpret_cast<const uint8_t*>(a.pool[of_v]) + row[i] * a.D + d);
          scale[i] = a.scales[of_v][row[i]];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int n = n0 + i * groups;
      if (!here || n >= a.N) continue;
      if constexpr (kCoded) decode8<TYPE>(q[i], scale[i], x[i]);
      st8<PAST>(reinterpret_cast<TE*>(a.dst[of_v]) + ((int64_t)n * a.heads + h) * a.D + d, x[i]);
    }
  }
}

template <bool WRITE> as_status move(const kc_cache* c, const KvMove& a, hipStream_t st) {
  // few tokens: as many lanes as there are rows
  const int groups = 64 >> a.lanes_log, quads = (2 * a.heads + 3) / 4;
  const bool few = (int64_t)a.N * quads <= (int64_t)groups * 1024;
  const int per_block = groups * (few ? 1 : 4);
  // a launch takes less than 2^32 threads along a dimension
  const int64_t most = (((int64_t)1 << 24) - 1) / quads * per_block;
  hipError_t e = hipSuccess;
  auto run = [&](auto* t, auto type) {
    using TE = typename std::remove_pointer<decltype(t)>::type;
    constexpr int TYPE = decltype(type)::value;
    // The dense side past the caches where it is more than they may keep for the next reader.  us, int8, rows of 256 MB through / past them:
    // write 104 / 97, read 115 / 63; of 128 MB 47 / 50 and 36 / 34; of 64 MB 25 / 27 and 20 / 19.
    const bool past = (int64_t)a.N * 2 * a.heads * a.D * sizeof(TE) > (int64_t)96 << 20;
    auto kfn = few ? kv_move_kernel<TE, TYPE, WRITE, 1, false> : past ? kv_move_kernel<TE, TYPE, WRITE, 4, true> : kv_move_kernel<TE, TYPE, WRITE, 4, false>;
    for (int64_t n0 = 0; n0 < a.N && e == hipSuccess; n0 += most) {
      KvMove p = a;
      p.N = (int32_t)(a.N - n0 < most ? a.N - n0 : most);
      p.seq += n0;
      p.pos += n0;
      for (int i = 0; i < 2; ++i) {
        if (WRITE) p.src[i] = reinterpret_cast<const TE*>(a.src[i]) + n0 * a.ld[i];
        else p.dst[i] = reinterpret_cast<TE*>(a.dst[i]) + n0 * a.heads * a.D;
      }
      hipLaunchKernelGGL(kfn, dim3((unsigned)((p.N + per_block - 1) / per_block * quads)), dim3(256), 0, st, p);
      e = hipGetLastError();
    }
  };
  auto any = [&](auto* t, auto same) {
    if (c->cache_type == KC_INT8) run(t, std::integral_constant<int, KC_INT8>{});
    else if (c->cache_type == KC_E4M3) run(t, std::integral_constant<int, KC_E4M3>{});
    else run(t, same);
  };
  if (c->dtype == AS_F32) any((float*)nullptr, std::integral_constant<int, KC_F32>{});
  else any((uint16_t*)nullptr, std::integral_constant<int, KC_BF16>{});
  return e == hipSuccess ? AS_OK : set_error(AS_ERR_HIP, "rows of the cache: %s", hipGetErrorString(e));
}

KvMove move_args(const kc_cache* c, int32_t N, const int32_t* seq, const int32_t* pos, const int32_t* table, const void* k_pages,
                 const void* v_pages, const float* k_scales, const float* v_scales) {
  KvMove a{};
  a.seq = seq;
  a.pos = pos;
  a.table = table;
  a.N = N;
  a.heads = c->heads;
  a.D = c->D;
  a.page = c->page;
  a.pages = c->pages;
  a.B = c->B;
  a.max_pages = c->max_pages;
  while (8 << a.lanes_log < c->D) ++a.lanes_log;
  a.pool[0] = const_cast<void*>(k_pages);
  a.pool[1] = const_cast<void*>(v_pages);
  a.scales[0] = const_cast<float*>(k_scales);
  a.scales[1] = const_cast<float*>(v_scales);
  return a;
}

}  // namespace
}  // namespace asx

using namespace asx;

extern "C" as_status kv_cache_write(const kc_cache* cache, int32_t N, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                                    const int32_t* seq, const int32_t* pos, const int32_t* page_table, void* k_pages, void* v_pages,
                                    float* k_scales, float* v_scales, void* hip_stream) {
  as_status rc = kv_check_cache(cache);
  if (rc != AS_OK) return rc;
  if (N < 1 || N > (1 << 24)) return set_error(AS_ERR_SHAPE, "kv_cache_write: N=%d", N);
  if (!k || !v || !seq || !pos) return set_error(AS_ERR_NULL, "kv_cache_write: a required pointer is NULL");
  rc = kv_check_pool(cache, k_pages, v_pages, k_scales, v_scales, page_table, "kv_cache_write");
  if (rc != AS_OK) return rc;
  for (int64_t ld : {ld_k, ld_v}) {
    if (ld < (int64_t)cache->heads * cache->D || ld >= (int64_t)1 << 32) return set_error(AS_ERR_SHAPE, "kv_cache_write: rows %lld elements apart", (long long)ld);
    if (ld * (cache->dtype == AS_F32 ? 4 : 2) % 16 != 0)
      return set_error(AS_ERR_ALIGN, "kv_cache_write: rows %lld elements apart do not start on 16 bytes", (long long)ld);
  }
  for (const void* p : {k, v, (const void*)seq, (const void*)pos})
    if (!kv_al16(p)) return set_error(AS_ERR_ALIGN, "kv_cache_write: a pointer is not 16-byte aligned");
  if (k_pages == v_pages || (k_scales && k_scales == v_scales))
    return set_error(AS_ERR_SHAPE, "kv_cache_write: keys and values would be written to the same places");
  KvMove a = move_args(cache, N, seq, pos, page_table, k_pages, v_pages, k_scales, v_scales);
  a.src[0] = k;
  a.src[1] = v;
  a.ld[0] = ld_k;
  a.ld[1] = ld_v;
  return move<true>(cache, a, reinterpret_cast<hipStream_t>(hip_stream));
}

extern "C" as_status kv_cache_read(const kc_cache* cache, int32_t N, const void* k_pages, const void* v_pages, const float* k_scales,
                                   const float* v_scales, const int32_t* seq, const int32_t* pos, const int32_t* page_table, void* k, void* v,
                                   void* hip_stream) {
  as_status rc = kv_check_cache(cache);
  if (rc != AS_OK) return rc;
  if (N < 1 || N > (1 << 24)) return set_error(AS_ERR_SHAPE, "kv_cache_read: N=%d", N);
  if (!k || !v || !seq || !pos) return set_error(AS_ERR_NULL, "kv_cache_read: a required pointer is NULL");
  rc = kv_check_pool(cache, k_pages, v_pages, k_scales, v_scales, page_table, "kv_cache_read");
  if (rc != AS_OK) return rc;
  for (const void* p : {(const void*)k, (const void*)v, (const void*)seq, (const void*)pos})
    if (!kv_al16(p)) return set_error(AS_ERR_ALIGN, "kv_cache_read: a pointer is not 16-byte aligned");
  KvMove a = move_args(cache, N, seq, pos, page_table, k_pages, v_pages, k_scales, v_scales);
  a.dst[0] = k;
  a.dst[1] = v;
  return move<false>(cache, a, reinterpret_cast<hipStream_t>(hip_stream));
}
