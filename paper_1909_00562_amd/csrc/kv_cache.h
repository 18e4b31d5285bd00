// What the cache's files share: checks of a cache's description and pointers, and division by products.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/kv_cache.h"

namespace asx {

constexpr int kKvTile = 16;   // tokens of a tile; pages are whole ones
inline bool kv_coded(int cache_type) { return cache_type == KC_INT8 || cache_type == KC_E4M3; }

as_status kv_check_cache(const kc_cache* c);
// the pool's pointers: what has to be there, and on 16 bytes
as_status kv_check_pool(const kc_cache* c, const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                        const int32_t* page_table, const char* what);
inline bool kv_al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Division of n < 2^24 by d <= 256 as a product: n (mul d - 2^32) < 2^32.  (2^32 itself, for d = 1, has no place in mul.)
struct KvMagic {
  uint32_t mul, itself;
};
inline KvMagic kv_magic(uint32_t d) {
  return d == 1 ? KvMagic{0, 0xffffffffu} : KvMagic{(uint32_t)((((uint64_t)1 << 32) + d - 1) / d), 0};
}
__device__ __forceinline__ uint32_t kv_div(uint32_t n, KvMagic m) { return __umulhi(n, m.mul) + (n & m.itself); }

}  // namespace asx
