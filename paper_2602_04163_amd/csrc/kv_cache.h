// The 8-bit key/value cache as the kernels see it (layout: include/bpdq.h).
#pragma once
#include "common.h"

namespace bpdq {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kKvTile = 64;                              // tokens per tile of the layout

// 16-byte chunk of a page and head's K that holds channels 16 c16 .. + 15 of slot t
__device__ __forceinline__ int kv_k_chunk(int t, int c16, int dim) {
  const int u = (t >> 2) & 3, g = (t >> 4) & 3, i = t & 3;
  return (t >> 6) * 4 * dim + (u * (dim >> 4) + c16) * 16 + 4 * g + i;
}
// and of its V that holds slots 16 s16 .. + 15 of channel d
__device__ __forceinline__ int kv_v_chunk(int s16, int d, int dim) {
  return (s16 >> 2) * 4 * dim + ((d >> 4) * 4 + (s16 & 3)) * 16 + (d & 15);
}

static inline bool kv_cache_ok(const bpdq_kv_cache* c) {
  return c && c->k && c->v && c->k_scale && c->v_scale && !(reinterpret_cast<uintptr_t>(c->k) & 15) &&
         !(reinterpret_cast<uintptr_t>(c->v) & 15) && !(reinterpret_cast<uintptr_t>(c->k_scale) & 3) &&
         !(reinterpret_cast<uintptr_t>(c->v_scale) & 3) && c->n_pages > 0 && c->n_kv > 0 && c->n_kv <= 65535 &&
         (c->page == 64 || c->page == 128 || c->page == 256) &&
         (c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 256);
}

}  // namespace bpdq
