// The 8-bit key/value cache: quantizing tokens as they are written, and reading them back.
//
// Per page and head, with amax the largest magnitude of the page's new tokens,
//   first slot new:  s = max(amax, 2^-96) / 127          else:  s' = s 2^j, smallest j >= 0 with amax <= 127 s 2^j
//   code = rint(x / s) + 128, and where the scale grew by 2^j the codes before become rint((code - 128) 2^-j) + 128.
// Growing by powers of two makes the rescaling of codes exact but for its one rounding, and the errors of repeated growth a
// geometric series: half a step from the last, a quarter of the present step from the one before and so on, below one step in all.
// With scales that grew by just what is needed, a code that a growth of less than half a step leaves where it is would drift by up
// to half a step per token.
//
// One work-group per page that is touched, head, and K or V: it alone reads and writes that scale and those codes.  K is
// kept by token (16 channels of a token are one 16-byte chunk), V by channel (16 tokens of a channel): V goes through LDS,
// where 4 x 4 bytes at a time are transposed by v_perm_b32.  (Pages are the unit because a scale's maximum and the codes that it rescales
// are a page's: no atomics, no second launch.)
//
// What bounds it: bytes, and for small calls the launch.  Measured (back to back on the same buffers): writing 4096 fp16 tokens of 8 heads of
// 128 moves 25 MB in 9.8 us (2.6 TB/s: a work-group loads, reduces over its page, then stores, and the call is one round of them),
// reading them back 25 MB in 8.0 us (3.1 TB/s); reading 37 sequences of up to 3777 tokens, 5 heads of 64, as floats moves 320 MB in
// 59 us (5.4 TB/s; a large copy reaches 5.3); one bf16 token for each of 16 sequences, 4 heads of 128, is written in 4.8 us, mostly latency.
#include "kv_cache.h"

namespace bpdq {

constexpr int kKvThreads = 256;
constexpr int kKvKeep = 2;
constexpr float kKvFloor = 0x1p-96f;

// 16 consecutive values as floats
template <typename T>
__device__ __forceinline__ void kv_load16(const T* __restrict__ p, bool vec, float (&x)[16]) {
  if (vec) {
    alignas(16) T raw[16];
#pragma unroll
    for (int q = 0; q < (int)sizeof(T); ++q) reinterpret_cast<u32x4_t*>(raw)[q] = reinterpret_cast<const u32x4_t*>(p)[q];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = (float)raw[e];
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = (float)p[e];
  }
}

__device__ __forceinline__ uint32_t kv_code(float x, float inv) {
  // a NaN (of a page whose scale is NaN) becomes the lower bound
  return (uint32_t)((int)fminf(fmaxf(rintf(x * inv), -127.f), 127.f) + 128);
}

__device__ __forceinline__ uint32_t kv_pack4(const float* x, float inv) {
  return kv_code(x[0], inv) | kv_code(x[1], inv) << 8 | kv_code(x[2], inv) << 16 | kv_code(x[3], inv) << 24;
}

// four codes under a scale that grew by 1 / shrink
__device__ __forceinline__ uint32_t kv_rescale4(uint32_t w, float shrink) {
  uint32_t out = 0;
#pragma unroll
  for (int b = 0; b < 4; ++b) out |= kv_code((float)((int)((w >> (8 * b)) & 255u) - 128), shrink) << (8 * b);
  return out;
}

// rows a, b, c, d of four bytes each to their columns
__device__ __forceinline__ void kv_transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&out)[4]) {
  const uint32_t t0 = __builtin_amdgcn_perm(b, a, 0x05010400u), t1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
  const uint32_t u0 = __builtin_amdgcn_perm(d, c, 0x05010400u), u1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
  out[0] = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
}

// Which slots of which page a work-group works on.  `there`: there are some.
struct KvSpan {
  long row;                                              // row of K or V of slot 0 (below 0 where the page began before)
  int lo, hi;                                            // slots lo .. hi - 1
  int phys;                                              // the page, or -1
  bool there;
};

__device__ __forceinline__ KvSpan kv_span(const bpdq_kv_cache& c, const int* __restrict__ table, int max_pages,
                                          const int* __restrict__ pos, const int* __restrict__ tok_start, int n_tok,
                                          int max_tok, int seq, int touch) {
  KvSpan s;
  const long p0 = pos[seq], first = tok_start[seq];
  long n = (long)tok_start[seq + 1] - first;
  n = n < max_tok ? n : max_tok;
  n = n < n_tok - first ? n : n_tok - first;
  s.there = false;
  if (p0 < 0 || first < 0 || n <= 0) return s;
  const long lp = p0 / c.page + touch, base = lp * c.page;
  s.lo = (int)(p0 > base ? p0 - base : 0);
  const long end = p0 + n - base;
  s.hi = (int)(end < c.page ? end : c.page);
  if (s.hi <= s.lo) return s;
  s.there = true;
  s.row = first + base - p0;
  const int id = lp < max_pages ? table[(long)seq * max_pages + lp] : -1;
  s.phys = id >= 0 && id < c.n_pages ? id : -1;
  return s;
}

constexpr int kv_lds_row(int dim) { return dim + 4; }     // bytes of a slot in LDS: slots 16 apart fall into other banks

// Two passes over the new tokens, one for amax and one for the codes.
template <typename T, int D>
__global__ __launch_bounds__(kKvThreads) void kv_write_kernel(bpdq_kv_cache c, const int* __restrict__ table, int max_pages,
                                                              const int* __restrict__ pos, const int* __restrict__ tok_start,
                                                              int n_tok, int max_tok, const T* __restrict__ K, long ldk,
                                                              const T* __restrict__ V, long ldv, int vec_k, int vec_v) {
  extern __shared__ uint8_t lds[];
  constexpr int kRow = kv_lds_row(D);
  const int tid = threadIdx.x;
  const int h = blockIdx.x % c.n_kv, touch = blockIdx.x / (2 * c.n_kv);
  const bool is_v = (blockIdx.x / c.n_kv) & 1;
  const KvSpan s = kv_span(c, table, max_pages, pos, tok_start, n_tok, max_tok, blockIdx.y, touch);
  if (!s.there || s.phys < 0) return;                    // uniform
  const T* src = (is_v ? V : K) + (long)h * D;
  const long ld = is_v ? ldv : ldk;
  const bool vec = is_v ? vec_v : vec_k;
  const long at = (long)s.phys * c.n_kv + h;
  u32x4_t* out = reinterpret_cast<u32x4_t*>((is_v ? c.v : c.k) + at * c.page * D);
  float* scale_at = (is_v ? c.v_scale : c.k_scale) + at;
  const int items = (s.hi - s.lo) * (D / 16);

  // the largest magnitude, as bits: a NaN is above an infinity, an infinity above every number
  const float old = s.lo > 0 ? *scale_at : 0.f;
  uint32_t most = 0;
  auto fetch = [&](int id, float (&x)[16]) {
    kv_load16(src + (s.row + s.lo + id / (D / 16)) * ld + 16 * (id % (D / 16)), vec, x);
  };
  auto look = [&](const float (&x)[16]) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t b = __builtin_bit_cast(uint32_t, x[e]) & 0x7fffffffu;
      most = most > b ? most : b;
    }
  };
  // a thread's first kKvKeep items (all of a page of 64 tokens of 128 channels) stay in registers, others are read again
  float kept[kKvKeep][16];
#pragma unroll
  for (int n = 0; n < kKvKeep; ++n)
    if (tid + n * kKvThreads < items) fetch(tid + n * kKvThreads, kept[n]);
#pragma unroll
  for (int n = 0; n < kKvKeep; ++n)
    if (tid + n * kKvThreads < items) look(kept[n]);
  for (int id = tid + kKvKeep * kKvThreads; id < items; id += kKvThreads) {
    float x[16];
    fetch(id, x);
    look(x);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t b = __shfl_xor(most, o, 64);
    most = most > b ? most : b;
  }
  __shared__ uint32_t wave_most[kKvThreads / 64];
  if ((tid & 63) == 0) wave_most[tid >> 6] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kKvThreads / 64; ++w) most = most > wave_most[w] ? most : wave_most[w];

  const float amax = __builtin_bit_cast(float, most);
  float scale, shrink = 1.f;
  bool grew = false;
  if (most >= 0x7f800000u) {
    scale = __builtin_nanf("");
  } else if (s.lo == 0) {
    scale = fmaxf(amax, kKvFloor) * (1.0f / 127.0f);
  } else {
    scale = old;
    const float limit = 127.f * old;
    if (amax > limit) {
      int e0, e1;
      const float m0 = frexpf(limit, &e0), m1 = frexpf(amax, &e1);
      const int up = e1 - e0 + (m1 > m0 ? 1 : 0);
      scale = ldexpf(old, up);
      shrink = ldexpf(1.f, -up);
      grew = true;
    }
  }
  if (tid == 0 && (s.lo == 0 || !(scale == old))) *scale_at = scale;
  const float inv = 1.f / scale;

  auto put = [&](int id, const float (&x)[16]) {
    const int t = s.lo + id / (D / 16), c16 = id % (D / 16);
    u32x4_t w;
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = kv_pack4(x + 4 * q, inv);
    if (!is_v) {
      out[kv_k_chunk(t, c16, D)] = w;
    } else {
      uint32_t* to = reinterpret_cast<uint32_t*>(lds + t * kRow + 16 * c16);
#pragma unroll
      for (int q = 0; q < 4; ++q) to[q] = w[q];
    }
  };
#pragma unroll
  for (int n = 0; n < kKvKeep; ++n)
    if (tid + n * kKvThreads < items) put(tid + n * kKvThreads, kept[n]);
  for (int id = tid + kKvKeep * kKvThreads; id < items; id += kKvThreads) {
    float x[16];
    fetch(id, x);
    put(id, x);
  }
  if (!is_v) {
    if (grew) {
      for (int id = tid; id < s.lo * (D / 16); id += kKvThreads) {
        u32x4_t* p = out + kv_k_chunk(id / (D / 16), id % (D / 16), D);
        u32x4_t w = *p;
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = kv_rescale4(w[q], shrink);
        *p = w;
      }
    }
    return;
  }
  __syncthreads();
  // 16 slots of four channels at a time
  const int s16_lo = grew ? 0 : s.lo / 16, s16_n = (s.hi + 15) / 16 - s16_lo;
  for (int id = tid; id < s16_n * (D / 4); id += kKvThreads) {
    const int s16 = s16_lo + id / (D / 4), d = 4 * (id % (D / 4));
    u32x4_t* p = out + kv_v_chunk(s16, d, D);
    u32x4_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t row[4], col[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = 16 * s16 + 4 * q + i;
        row[i] = t >= s.lo && t < s.hi ? *reinterpret_cast<const uint32_t*>(lds + t * kRow + d) : 0u;
      }
      kv_transpose4(row[0], row[1], row[2], row[3], col);
#pragma unroll
      for (int m = 0; m < 4; ++m) w[m][q] = col[m];
    }
    if (16 * s16 < s.lo || 16 * s16 + 16 > s.hi) {       // slots that are there already, or are not yet
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t fresh = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = 16 * s16 + 4 * q + i;
          if (t >= s.lo && t < s.hi) fresh |= 0xffu << (8 * i);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          uint32_t b = p[m][q];
          if (grew) b = kv_rescale4(b, shrink);
          w[m][q] = (w[m][q] & fresh) | (b & ~fresh);
        }
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) p[m] = w[m];
  }
}

// One work-group per page, head, and K or V as above; V is transposed through LDS, so that both ways memory is asked for whole lines.
template <typename T, int D>
__global__ __launch_bounds__(kKvThreads) void kv_read_kernel(bpdq_kv_cache c, const int* __restrict__ table, int max_pages,
                                                             const int* __restrict__ pos, const int* __restrict__ tok_start,
                                                             int n_tok, int max_tok, T* __restrict__ K, long ldk,
                                                             T* __restrict__ V, long ldv, int vec_k, int vec_v) {
  extern __shared__ uint8_t lds[];
  constexpr int kRow = kv_lds_row(D);
  const int tid = threadIdx.x;
  const int h = blockIdx.x % c.n_kv, touch = blockIdx.x / (2 * c.n_kv);
  const bool is_v = (blockIdx.x / c.n_kv) & 1;
  const KvSpan s = kv_span(c, table, max_pages, pos, tok_start, n_tok, max_tok, blockIdx.y, touch);
  if (!s.there) return;                                  // uniform
  T* dst = (is_v ? V : K) + (long)h * D;
  const long ld = is_v ? ldv : ldk;
  const bool vec = is_v ? vec_v : vec_k;
  const long at = (long)(s.phys < 0 ? 0 : s.phys) * c.n_kv + h;
  const u32x4_t* in = reinterpret_cast<const u32x4_t*>((is_v ? c.v : c.k) + at * c.page * D);
  const float scale = s.phys < 0 ? 0.f : (is_v ? c.v_scale : c.k_scale)[at];

  // codes to LDS by slot, as they lie in the cache
  if (s.phys >= 0 && is_v) {
    const int s16_lo = s.lo / 16, s16_n = (s.hi + 15) / 16 - s16_lo;
    for (int id = tid; id < s16_n * (D / 4); id += kKvThreads) {
      const int s16 = s16_lo + id / (D / 4), d = 4 * (id % (D / 4));
      const u32x4_t* p = in + kv_v_chunk(s16, d, D);
      const u32x4_t w[4] = {p[0], p[1], p[2], p[3]};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t row[4];
        kv_transpose4(w[0][q], w[1][q], w[2][q], w[3][q], row);
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(lds + (16 * s16 + 4 * q + i) * kRow + d) = row[i];
      }
    }
  } else if (s.phys >= 0) {
    const int tile_lo = s.lo / kKvTile, tile_n = (s.hi + kKvTile - 1) / kKvTile - tile_lo;
    for (int id = tid; id < tile_n * 4 * D; id += kKvThreads) {
      const int at = id % (4 * D), c16 = at / 16 % (D / 16);
      const int t = (tile_lo + id / (4 * D)) * kKvTile + 16 * (at / 4 % 4) + 4 * (at / D) + at % 4;
      if (t < s.lo || t >= s.hi) continue;
      const u32x4_t w = in[(tile_lo * 4 * D) + id];
      uint32_t* to = reinterpret_cast<uint32_t*>(lds + t * kRow + 16 * c16);
#pragma unroll
      for (int q = 0; q < 4; ++q) to[q] = w[q];
    }
  }
  __syncthreads();
  // and out, 16 bytes a lane, consecutive lanes consecutive channels
  constexpr int kVec = 16 / sizeof(T);
  for (int id = tid; id < (s.hi - s.lo) * (D / kVec); id += kKvThreads) {
    const int t = s.lo + id / (D / kVec), d = kVec * (id % (D / kVec));
    alignas(16) T out[kVec];
#pragma unroll
    for (int q = 0; q < kVec / 4; ++q) {
      const uint32_t w = s.phys >= 0 ? *reinterpret_cast<const uint32_t*>(lds + t * kRow + d + 4 * q) : 0x80808080u;
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * q + e] = (T)((float)((int)((w >> (8 * e)) & 255u) - 128) * scale);
    }
    T* to = dst + (s.row + t) * ld + d;
    if (vec) {
      *reinterpret_cast<u32x4_t*>(to) = *reinterpret_cast<const u32x4_t*>(out);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) to[e] = out[e];
    }
  }
}

// Pages of a sequence that n tokens from anywhere in a page can touch.
static int kv_touched(int n, int page) { return (int)(((long)n + page - 2) / page) + 1; }

static bool kv_vec(const void* p, long ld, size_t size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (size_t)ld * size % 16 == 0;
}

template <typename T, int D>
static int kv_launch(bool write, const bpdq_kv_cache& c, const int* table, int max_pages, int n_seq, const int* pos,
                     const int* tok_start, int n_tok, int max_tok, void* K, long ldk, void* V, long ldv, hipStream_t stream) {
  const int touched = kv_touched(max_tok, c.page);
  const dim3 grid((unsigned)touched * 2 * c.n_kv, n_seq);
  const size_t bytes = (size_t)c.page * kv_lds_row(D);
  const int vec_k = kv_vec(K, ldk, sizeof(T)), vec_v = kv_vec(V, ldv, sizeof(T));
  if (write) {
    BPDQ_HIP_TRY((bpdq_lds_limit<&kv_write_kernel<T, D>>(256 * kv_lds_row(D))));
    hipLaunchKernelGGL((kv_write_kernel<T, D>), grid, dim3(kKvThreads), bytes, stream, c, table, max_pages, pos, tok_start, n_tok,
                       max_tok, static_cast<const T*>(K), ldk, static_cast<const T*>(V), ldv, vec_k, vec_v);
  } else {
    BPDQ_HIP_TRY((bpdq_lds_limit<&kv_read_kernel<T, D>>(256 * kv_lds_row(D))));
    hipLaunchKernelGGL((kv_read_kernel<T, D>), grid, dim3(kKvThreads), bytes, stream, c, table, max_pages, pos, tok_start, n_tok,
                       max_tok, static_cast<T*>(K), ldk, static_cast<T*>(V), ldv, vec_k, vec_v);
  }
  BPDQ_LAUNCH_CHECK();
  return 0;
}

template <typename T>
static int kv_by_dim(bool write, const bpdq_kv_cache& c, const int* table, int max_pages, int n_seq, const int* pos,
                     const int* tok_start, int n_tok, int max_tok, void* K, long ldk, void* V, long ldv, hipStream_t stream) {
  switch (c.head_dim) {
    case 64: return kv_launch<T, 64>(write, c, table, max_pages, n_seq, pos, tok_start, n_tok, max_tok, K, ldk, V, ldv, stream);
    case 128: return kv_launch<T, 128>(write, c, table, max_pages, n_seq, pos, tok_start, n_tok, max_tok, K, ldk, V, ldv, stream);
    default: return kv_launch<T, 256>(write, c, table, max_pages, n_seq, pos, tok_start, n_tok, max_tok, K, ldk, V, ldv, stream);
  }
}

static int kv_move(bool write, const bpdq_kv_cache* c, const int* table, int max_pages, int n_seq, const int* pos,
                   const int* tok_start, int n_tok, int max_tok, void* K, long ldk, void* V, long ldv, int dtype, void* stream_) {
  if (!kv_cache_ok(c)) return -1;
  if (max_pages <= 0) return -3;
  if (n_seq < 0 || n_seq > 65535) return -4;
  if (n_tok < 0) return -7;
  if (max_tok < 0) return -8;
  if (dtype != BPDQ_F32 && dtype != BPDQ_F16 && dtype != BPDQ_BF16) return -13;
  if (n_seq == 0 || n_tok == 0 || max_tok == 0) return 0;
  const long row = (long)c->n_kv * c->head_dim;
  const uintptr_t odd = dtype == BPDQ_F32 ? 3 : 1;
  if (!table) return -2;
  if (!pos) return -5;
  if (!tok_start) return -6;
  if (!K || (reinterpret_cast<uintptr_t>(K) & odd)) return -9;
  if (ldk < row) return -10;
  if (!V || (reinterpret_cast<uintptr_t>(V) & odd)) return -11;
  if (ldv < row) return -12;
  if ((long)kv_touched(max_tok, c->page) * 2 * c->n_kv * kKvThreads > 0xffffffffL) return -8;    // threads along the grid's x
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (dtype == BPDQ_F32)
    return kv_by_dim<float>(write, *c, table, max_pages, n_seq, pos, tok_start, n_tok, max_tok, K, ldk, V, ldv, stream);
  if (dtype == BPDQ_F16)
    return kv_by_dim<_Float16>(write, *c, table, max_pages, n_seq, pos, tok_start, n_tok, max_tok, K, ldk, V, ldv, stream);
  return kv_by_dim<__bf16>(write, *c, table, max_pages, n_seq, pos, tok_start, n_tok, max_tok, K, ldk, V, ldv, stream);
}

}  // namespace bpdq

extern "C" int bpdq_kv_write(const bpdq_kv_cache* cache, const int* page_table, int max_pages, int n_seq, const int* pos,
                             const int* tok_start, int n_tok, int max_tok, const void* K, long ldk, const void* V, long ldv,
                             int dtype, void* stream) {
  return bpdq::kv_move(true, cache, page_table, max_pages, n_seq, pos, tok_start, n_tok, max_tok, const_cast<void*>(K), ldk,
                       const_cast<void*>(V), ldv, dtype, stream);
}

extern "C" int bpdq_kv_read(const bpdq_kv_cache* cache, const int* page_table, int max_pages, int n_seq, const int* pos,
                            const int* tok_start, int n_tok, int max_tok, void* K, long ldk, void* V, long ldv, int dtype,
                            void* stream) {
  return bpdq::kv_move(false, cache, page_table, max_pages, n_seq, pos, tok_start, n_tok, max_tok, K, ldk, V, ldv, dtype, stream);
}
