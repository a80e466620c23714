// What the kernels of the key-value cache share: where a token's rows lie, and the 8-bit forms of a row.
//
// K and V of the cache are [n_pages, hkv, page_size, d]: the tokens of a page lie next to each other head by head, so that the
// attention of one head streams page_size * d elements at a time.  A "row" is the d elements of one token and head; its index
// counts them all, (page * hkv + head) * page_size + place in the page, and its scale (8-bit forms) has the same index.
#pragma once
#include "va_internal.h"
#include "va_mfma_common.h"

namespace va {

struct F32 {  // beside Bf16 and F16
  typedef float elem;
};
// Element types of the cache in 8 bits; kTop: what a row's largest element is stored as; kMostScale: the largest scale whose
// product with it is finite (that of the largest fp32 number, rounded to nearest, may be half a step above).
struct I8 {
  typedef int8_t elem;
  static constexpr float kTop = 127.f;
  static constexpr float kMostScale = (float)(3.4028234663852886e38 / 127 * (1 - 0x1p-24));
};
struct E4m3 {
  typedef uint8_t elem;
  static constexpr float kTop = 448.f;
  static constexpr float kMostScale = (float)(3.4028234663852886e38 / 448 * (1 - 0x1p-24));
};
template <class C> struct is_8bit { static constexpr bool value = false; };
template <> struct is_8bit<I8> { static constexpr bool value = true; };
template <> struct is_8bit<E4m3> { static constexpr bool value = true; };

// Pages of the sequences of one call.
struct PageMap {
  const int32_t *table;
  int64_t stride;      // entries from one sequence's to the next's
  int32_t n_seqs, n_pages, hkv, capacity;  // capacity: tokens that a sequence's entries reach, max_pages * page_size
  FastDiv page;        // page_size
};
static inline PageMap page_map(const va_kv_cache &c) {
  return {c.page_table, c.table_stride, c.n_seqs, c.n_pages, c.hkv, c.max_pages * c.page_size, fast_div(c.page_size)};
}

// Row of head 0 of a token's place in the cache, or -1 where it has none: no such sequence, a position that the table does not
// reach, or an entry that is no page.  The row of head g is page_size * g behind it.
__device__ __forceinline__ int place_of(const PageMap &map, long long seq, long long position) {
  if (seq < 0 || seq >= map.n_seqs || position < 0 || position >= map.capacity) return -1;
  const int p = (int)position, at = p / map.page;
  const int id = map.table[seq * map.stride + at];
  return (uint32_t)id < (uint32_t)map.n_pages ? id * (int)(map.hkv * map.page.d) + (p - at * (int)map.page.d) : -1;
}

__device__ __forceinline__ float e4m3_to_f32(uint8_t x) {
  return __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false)[0];
}
__device__ __forceinline__ float cached_to_f32(I8, int8_t x) { return (float)x; }
__device__ __forceinline__ float cached_to_f32(E4m3, uint8_t x) { return e4m3_to_f32(x); }
template <class C> __device__ __forceinline__ float cached_to_f32(C, typename C::elem x) { return (float)x; }

}  // namespace va
