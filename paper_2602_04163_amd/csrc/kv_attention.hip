// Attention of new tokens over the 8-bit key/value cache:
//   out_r = sum_t p_t v_t / l,   p_t = exp(z_t - m),  z_t = scale <q_r, k_t>,  m = max z_t,  l = sum p_t
// in one pass over the cache with the running maximum and sum: after a tile of 64 tokens m' = max(m, tile), and l and the sums
// of p v are scaled by exp(m - m') before the tile's terms are added.
//
// A row r of a work item is a (query, head) pair of one key head: the G = n_q / n_kv heads that share it and, where a sequence
// brings several tokens, those tokens too, so that the cache is read once for all of them.
//
// Products.  Everything is computed transposed, S^T = K Q^T and O^T = V^T P^T: a lane then holds scores of one row (column
// l % 16 of the 16 x 16 tiles) and 16 tokens of a tile (16 (l / 16) ..), which is at the same time the operand layout that the
// second product wants of P^T, so P never leaves its registers, and a row's maximum and sum cross lanes twice only.  The token
// order inside a tile and the channel order inside the first product are free; the cache's layout is the one in which every load is 16 bytes
// a lane and 1 KB of consecutive bytes a wavefront.  A code byte becomes an fp16 by v_perm_b32 with 0x64 (1024 + code) and a
// packed subtraction of 1152, both exact.  The scale of K multiplies the scores, that of V a tile's share of O, in fp32.
//
// Work-group: four wavefronts that take the tiles of a chunk in turn, each with its own m, l and O, joined in LDS in a fixed
// order.  Long caches are cut into chunks, whose unnormalised O, m and l go to the workspace; a second launch joins them.
//
// What bounds it: single tokens read the cache once, 2 head_dim bytes per token and key head.  131071 fp16 tokens of 8 key heads of 128 (268 MB, 64
// heads) take 55 us and 6 us for the join (4.9 and 4.4 TB/s; a large copy reaches 5.3), 32 sequences of 1 to 16384 tokens (538 MB) 115 and 9
// (4.7 and 4.3), and 165 in all with 17 to 32 rows (four or five tokens a sequence); 1000 tokens of 4 key heads 11 us, the latency of four tiles in a
// row in a wavefront.  Prompts: see below.
#include "kv_cache.h"

namespace bpdq {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / 64;
constexpr int kAttnMostChunks = 512;                     // of a work item
constexpr int kAttnMostKv = 1 << 30;                     // a position (from -2^24 on) less a window, and a tile's end, are ints
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct AttnArgs {
  bpdq_kv_cache c;
  const int* table;
  const int* kv_len;
  const int* q_start;
  const void* q;
  void* out;
  float* lse;
  float* part;                                           // [item][chunk][rows][dim] sums, then [item][chunk][rows][2] m, l
  long ldq, ldo;
  int max_pages, n_tok, max_q, max_kv, n_q, group;
  int causal, window;
  int page_shift;                                        // tiles of a page, as a power of two
  int vec_q, vec_o;                                      // whether Q goes by 16 bytes, and out by four values
  int q_tiles, n_chunk, chunk_tiles;
  float scale;
};

// One work item: rows r0 .. of a sequence and key head, and the tiles of the cache that any of them sees.
struct AttnItem {
  int first, q_len, rows, r0, kv;
  int tile_lo, tile_hi;                                  // tiles tile_lo .. tile_hi - 1
  bool there;
};

template <int ROWS>
__device__ __forceinline__ AttnItem attn_item(const AttnArgs& a, int seq, int q_tile) {
  AttnItem it;
  it.first = a.q_start[seq];
  long n = (long)a.q_start[seq + 1] - it.first;
  n = n < a.max_q ? n : a.max_q;
  n = n < (long)a.n_tok - it.first ? n : (long)a.n_tok - it.first;
  it.there = false;
  if (it.first < 0 || n <= 0) return it;
  it.q_len = (int)n;
  it.rows = it.q_len * a.group;
  it.r0 = q_tile * ROWS;
  if (it.r0 >= it.rows) return it;
  it.there = true;
  int kv = a.kv_len[seq];
  kv = kv < 0 ? 0 : kv;
  it.kv = kv < a.max_kv ? kv : a.max_kv;
  const int last = (it.rows < it.r0 + ROWS ? it.rows : it.r0 + ROWS) - 1;
  const int off = it.kv - it.q_len;
  int hi = it.kv - 1, lo = 0;
  if (a.causal) hi = off + last / a.group < hi ? off + last / a.group : hi;
  if (a.window > 0) lo = off + it.r0 / a.group - a.window + 1 > 0 ? off + it.r0 / a.group - a.window + 1 : 0;
  it.tile_lo = lo / kKvTile;
  it.tile_hi = hi >= lo ? hi / kKvTile + 1 : it.tile_lo;
  return it;
}

__device__ __forceinline__ int attn_chunks(const AttnItem& it, int chunk_tiles) {
  const int n = bpdq_ceil_div(it.tile_hi - it.tile_lo, chunk_tiles);
  return n > 0 ? n : 1;
}

// eight codes (bytes of two words) as fp16
__device__ __forceinline__ f16x8_t attn_codes(uint32_t a, uint32_t b) {
  const f16x2_t zero = {(_Float16)1152.f, (_Float16)1152.f};
  auto two = [&](uint32_t bytes, uint32_t which) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, bytes, which)) - zero);
  };
  return __builtin_bit_cast(f16x8_t, u32x4_t{two(a, 0x04010400u), two(a, 0x04030402u), two(b, 0x04010400u), two(b, 0x04030402u)});
}

template <typename T>
__device__ __forceinline__ void attn_store4(T* to, f32x4_t v, bool vec) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  const T4 out = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  if (vec) {
    *reinterpret_cast<T4*>(to) = out;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) to[e] = out[e];
  }
}

// T: type of Q and out;  D: head dimension;  NQ: tiles of 16 rows.
template <typename T, int D, int NQ>
__global__ __launch_bounds__(kAttnThreads) void attn_rows_kernel(AttnArgs a) {
  constexpr int ROWS = 16 * NQ, C = D / 64, DT = D / 16, kAcc = D + 4;
  __shared__ float acc_s[ROWS * kAcc];
  __shared__ float m_s[kAttnWaves][ROWS], l_s[kAttnWaves][ROWS];
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int chunk = blockIdx.x % a.n_chunk;
  const int item = blockIdx.x / a.n_chunk;               // (head, query tile)
  const int h = item % a.c.n_kv, q_tile = item / a.c.n_kv, seq = blockIdx.y;
  const int page_shift = a.page_shift, page_mask = (1 << page_shift) - 1;           // tiles of a page
  const AttnItem it = attn_item<ROWS>(a, seq, q_tile);
  if (!it.there) return;                                 // uniform
  const int n_chunk = attn_chunks(it, a.chunk_tiles);
  if (chunk >= n_chunk) return;
  const int t_begin = it.tile_lo + chunk * a.chunk_tiles;
  const int t_end = it.tile_hi < t_begin + a.chunk_tiles ? it.tile_hi : t_begin + a.chunk_tiles;

  // the rows' queries as operands: channel 64 c + 16 quarter + 8 s + j is k = 8 quarter + j of product (c, s)
  f16x8_t qf[NQ][C][2];
  float q_scale[NQ];                                     // of the scores, to base 2
  int see_lo[NQ], see_hi[NQ];                            // tokens that the lane's row sees: see_lo <= t < see_hi
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = it.r0 + 16 * n + col;
    const bool on = r < it.rows;
    const int i = (on ? r : 0) / a.group, head = h * a.group + (on ? r : 0) % a.group;
    const T* q = static_cast<const T*>(a.q) + (long)(it.first + i) * a.ldq + (long)head * D;
    float most = 0.f;
    alignas(16) T x[C][16];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const T* from = q + 64 * c + 16 * quarter;
      if (a.vec_q) {
#pragma unroll
        for (int e = 0; e < 2; ++e) reinterpret_cast<u32x4_t*>(x[c])[e] = reinterpret_cast<const u32x4_t*>(from)[e];
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[c][e] = from[e];
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) most = fmaxf(most, fabsf((float)x[c][e]));
    float f = 1.f, back = 1.f;
    if constexpr (sizeof(T) == 2 && !__is_same(T, _Float16)) {
      most = fmaxf(most, __shfl_xor(most, 16, 64));
      most = fmaxf(most, __shfl_xor(most, 32, 64));
      if (most > 0.f && most < __builtin_huge_valf()) {  // into [2^14, 2^15)
        int e;
        (void)frexpf(most, &e);
        e = 15 - e < 126 ? 15 - e : 126;
        f = ldexpf(1.f, e);
        back = ldexpf(1.f, -e);
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) qf[n][c][e / 8][e % 8] = (_Float16)((float)x[c][e] * f);
    q_scale[n] = back * (a.scale * kLog2e);
    const int p = it.kv - it.q_len + i;
    see_lo[n] = a.window > 0 ? p - a.window + 1 : 0;
    see_hi[n] = !on ? 0 : a.causal && p + 1 < it.kv ? p + 1 : it.kv;
  }

  f32x4_t o[NQ][DT];
  float m[NQ], l[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m[n] = -__builtin_huge_valf();
    l[n] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[n][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  // A tile's K is requested while the tile before is worked on, its V before its own scores: some 8 KB of a wavefront are always on
  // their way.  Pages outside the cache are stepped over.
  const int* row_of_table = a.table + (long)seq * a.max_pages;
  auto page_from = [&](int& tile) {                      // of the next tile from `tile` on that is there, or -1
    for (; tile < t_end; tile += kAttnWaves) {
      const int id = row_of_table[tile >> page_shift];
      if (id >= 0 && id < a.c.n_pages) return id;
    }
    return -1;
  };
  u32x4_t kw[4 * C], vw[DT];
  long at = 0;                                           // page and head
  float k_scale = 0.f, v_scale = 0.f;
  auto load_k = [&](int id, int tile) {
    at = (long)id * a.c.n_kv + h;
    const u32x4_t* from = reinterpret_cast<const u32x4_t*>(a.c.k + at * a.c.page * D + (long)(tile & page_mask) * kKvTile * D) + lane;
#pragma unroll
    for (int n = 0; n < 4 * C; ++n) kw[n] = from[n * 64];
  };
  int tile = t_begin + wave;
  int id = page_from(tile);
  if (id >= 0) load_k(id, tile);
  while (id >= 0) {
    {
      const u32x4_t* from = reinterpret_cast<const u32x4_t*>(a.c.v + at * a.c.page * D + (long)(tile & page_mask) * kKvTile * D) + lane;
#pragma unroll
      for (int d = 0; d < DT; ++d) vw[d] = from[d * 64];
    }
    k_scale = a.c.k_scale[at];
    v_scale = a.c.v_scale[at];
    int tile_next = tile + kAttnWaves;
    const int id_next = page_from(tile_next);
    f32x4_t s[NQ][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n][u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const u32x4_t w = kw[u * C + c];
        const f16x8_t k0 = attn_codes(w[0], w[1]), k1 = attn_codes(w[2], w[3]);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          s[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qf[n][c][0], s[n][u], 0, 0, 0);
          s[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qf[n][c][1], s[n][u], 0, 0, 0);
        }
      }
    }
    if (id_next >= 0) load_k(id_next, tile_next);
    // values of a page whose scale is not finite reach the rows that see them, and no others: by the probabilities
    const bool bad = !(fabsf(v_scale) < __builtin_huge_valf());
    if (bad) v_scale = 1.f;
    f16x8_t p[NQ][2];
    float fade[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const float f = k_scale * q_scale[n];
      const int t0 = tile * kKvTile + 16 * quarter;
      float top = m[n];
      bool seen[4][4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + 4 * u + i;
          seen[u][i] = t >= see_lo[n] && t < see_hi[n];
          s[n][u][i] = seen[u][i] ? s[n][u][i] * f : -__builtin_huge_valf();
          top = fmaxf(top, s[n][u][i]);
        }
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float base = top == -__builtin_huge_valf() ? 0.f : top;
      fade[n] = __builtin_amdgcn_exp2f(m[n] - base);
      m[n] = top;
      l[n] *= fade[n];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float e = __builtin_amdgcn_exp2f(s[n][u][i] - base);
          if (bad && seen[u][i]) e = __builtin_nanf("");
          l[n] += e;
          p[n][u / 2][4 * (u % 2) + i] = (_Float16)e;
        }
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const u32x4_t w = vw[d];
      const f16x8_t v0 = attn_codes(w[0], w[1]), v1 = attn_codes(w[2], w[3]);
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        f32x4_t pv = {0.f, 0.f, 0.f, 0.f};
        pv = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[n][0], pv, 0, 0, 0);
        pv = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[n][1], pv, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][d][i] = fmaf(o[n][d][i], fade[n], v_scale * pv[i]);
      }
    }
    tile = tile_next;
    id = id_next;
  }

  // join the wavefronts
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    l[n] += __shfl_xor(l[n], 16, 64);
    l[n] += __shfl_xor(l[n], 32, 64);
    if (lane < 16) {
      m_s[wave][16 * n + col] = m[n];
      l_s[wave][16 * n + col] = l[n];
    }
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float top = m_s[0][16 * n + col];
#pragma unroll
    for (int w = 1; w < kAttnWaves; ++w) top = fmaxf(top, m_s[w][16 * n + col]);
    // a wavefront that saw nothing has zero sums (or a NaN, which stays)
    const float f = m[n] == -__builtin_huge_valf() ? 1.f : __builtin_amdgcn_exp2f(m[n] - top);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][d][i] *= f;
  }
  for (int w = 0; w < kAttnWaves; ++w) {
    if (wave == w) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          f32x4_t* at = reinterpret_cast<f32x4_t*>(acc_s + (16 * n + col) * kAcc + 16 * d + 4 * quarter);
          *at = w ? *at + o[n][d] : o[n][d];
        }
    }
    __syncthreads();
  }
  const int out_rows = it.rows - it.r0 < ROWS ? it.rows - it.r0 : ROWS;
  const long slot = (((long)seq * a.q_tiles + q_tile) * a.c.n_kv + h) * a.n_chunk + chunk;
  const long n_slot = (long)gridDim.y * a.q_tiles * a.c.n_kv * a.n_chunk;
  for (int id = tid; id < out_rows * (D / 4); id += kAttnThreads) {
    const int r = id / (D / 4), d = 4 * (id % (D / 4));
    float top = m_s[0][r];
#pragma unroll
    for (int w = 1; w < kAttnWaves; ++w) top = fmaxf(top, m_s[w][r]);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w)
      sum += l_s[w][r] * (m_s[w][r] == -__builtin_huge_valf() ? 1.f : __builtin_amdgcn_exp2f(m_s[w][r] - top));
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(acc_s + r * kAcc + d);
    if (n_chunk > 1) {
      *reinterpret_cast<f32x4_t*>(a.part + (slot * ROWS + r) * D + d) = v;
      if (d == 0) {
        float* ml = a.part + n_slot * ROWS * D + (slot * ROWS + r) * 2;
        ml[0] = top;
        ml[1] = sum;
      }
    } else {
      const int i = (it.r0 + r) / a.group, head = h * a.group + (it.r0 + r) % a.group;
      T* to = static_cast<T*>(a.out) + (long)(it.first + i) * a.ldo + (long)head * D + d;
      const float f = sum == 0.f ? 0.f : 1.f / sum;
      attn_store4(to, v * f, a.vec_o);
      if (a.lse && d == 0)
        a.lse[(long)(it.first + i) * a.n_q + head] = sum == 0.f ? -__builtin_huge_valf() : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
}

// Many rows (prompts): products of 32 x 32, and K and V of a tile turned into fp16 once for the work-group's 128 rows, in LDS, in operand
// order.  A wavefront owns 32 rows; S^T = K Q^T and O^T = V^T P^T as above (row a of the first product's operand is the token that makes a lane's
// scores the second one's operand: 16 s + 8 j + 4 h + i <-> token 16 s + 8 h + 4 j + i of 32).
//
// 4096 bf16 tokens, 28 heads of 128 on 4 key heads, causal: 150 to 164 us, 735 to 800 TFLOP/s (a library product reaches 1450; the matrix
// instructions of the same work take 44 % of the time, and the exponentials beside them share the SIMD's issue).
// What bounds it is the vector unit, so the softmax is kept to a multiply-add, an exponential, a maximum, a sum and half a conversion per score:
//  - running maxima are followed lazily: sums are rescaled only when a row's terms grow by more than 2^8 of the reference;
//  - the scale of V goes into the exponent, so P V adds up in the accumulators.  A row has two references for that: m, the largest z, for the sum of
//    its p, and mv, the largest z + log2(scale of V), for its sums of p v.  The terms of the product are 2^7 exp2(z + log2(scale) - mv): up
//    to 2^15 of fp16's 2^16, and denormal, with an absolute error, below 2^-21 of the largest p scale of the tokens that the row sees.  One factor per
//    tile, undo, turns a tile's sum of these terms into its share of l.  Both references are of what the row itself sees, and only ever rise, so
//    scales of V however far apart neither overflow a sum nor hide another page's terms: what is lost is small beside the row's largest term.
//    (Where a tile's scale is so small that its terms would leave the range of fp32, below 2^-57, they are held at that: the product takes
//    zeros, which is what they are in fp16, and l its whole share.)
// The scale of scores must not be negative for the maximum: its sign goes into Q.
template <typename T, int D>
struct AttnPrompt {
  static constexpr int kRows = 128, kKs = D / 16, kDt = D / 32;
  static constexpr int kBuf = kKvTile * D * 2;           // bytes of a tile's K, and of its V, as fp16
  static constexpr int kChunks = kKvTile * D / 16 / kAttnThreads;   // 16-byte chunks of K, and of V, of a thread
  static constexpr size_t kLds = 4 * kBuf;               // two of each
};

template <typename T, int D>
__global__ __launch_bounds__(kAttnThreads, D == 256 ? 1 : 2) void attn_prompt_kernel(AttnArgs a) {
  typedef AttnPrompt<T, D> P;
  constexpr int ROWS = P::kRows, kKs = P::kKs, kDt = P::kDt, kChunks = P::kChunks;
  extern __shared__ uint4 lds_raw[];
  char* lds = reinterpret_cast<char*>(lds_raw);
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int chunk = blockIdx.x % a.n_chunk;
  const int item = blockIdx.x / a.n_chunk;
  // the last queries see most: they go first
  const int h = item % a.c.n_kv, q_tile = a.q_tiles - 1 - item / a.c.n_kv, seq = blockIdx.y;
  const int page_shift = a.page_shift, page_mask = (1 << page_shift) - 1;           // tiles of a page
  const AttnItem it = attn_item<ROWS>(a, seq, q_tile);
  if (!it.there) return;                                 // uniform
  const int n_chunk = attn_chunks(it, a.chunk_tiles);
  if (chunk >= n_chunk) return;
  const int t_begin = it.tile_lo + chunk * a.chunk_tiles;
  const int t_end = it.tile_hi < t_begin + a.chunk_tiles ? it.tile_hi : t_begin + a.chunk_tiles;

  // the wavefront's rows: operands, and what they see
  const int r = it.r0 + 32 * wave + col;
  const bool on = r < it.rows;
  const int i = (on ? r : 0) / a.group, head = h * a.group + (on ? r : 0) % a.group;
  f16x8_t qf[kKs];
  float q_scale;
  {
    const T* q = static_cast<const T*>(a.q) + (long)(it.first + i) * a.ldq + (long)head * D + 8 * half;
    alignas(16) T x[kKs][8];
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < kKs; ++k) {
      if (a.vec_q) {
        *reinterpret_cast<u32x4_t*>(x[k]) = *reinterpret_cast<const u32x4_t*>(q + 16 * k);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[k][e] = q[16 * k + e];
      }
    }
#pragma unroll
    for (int k = 0; k < kKs; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf((float)x[k][e]));
    float f = a.scale < 0.f ? -1.f : 1.f, back = 1.f;
    if constexpr (!__is_same(T, _Float16)) {
      most = fmaxf(most, __shfl_xor(most, 32, 64));
      if (most > 0.f && most < __builtin_huge_valf()) {  // into [2^14, 2^15)
        int e;
        (void)frexpf(most, &e);
        e = 15 - e < 126 ? 15 - e : 126;
        f *= ldexpf(1.f, e);
        back = ldexpf(1.f, -e);
      }
    }
#pragma unroll
    for (int k = 0; k < kKs; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[k][e] = (_Float16)((float)x[k][e] * f);
    q_scale = back * (fabsf(a.scale) * kLog2e);
  }
  const int at_q = it.kv - it.q_len + i;
  const int see_lo = a.window > 0 ? at_q - a.window + 1 : 0;
  const int see_hi = !on ? 0 : a.causal && at_q + 1 < it.kv ? at_q + 1 : it.kv;
  // of all the wavefront's rows: tokens that all see
  int all_lo = on ? see_lo : 0, all_hi = on ? see_hi : 0x7fffffff;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const int lo = __shfl_xor(all_lo, o, 64), hi = __shfl_xor(all_hi, o, 64);
    all_lo = all_lo > lo ? all_lo : lo;
    all_hi = all_hi < hi ? all_hi : hi;
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);

  // Pages and scales of the tiles from `known` on, one to a lane; -1 where there is nothing to be seen (behind the last tile, or a page
  // outside the cache).
  const int* row_of_table = a.table + (long)seq * a.max_pages;
  int known = 0, page_of = -1;
  float k_scale_of = 0.f, v_scale_of = 0.f;
  auto learn = [&](int tile) {
    known = tile;
    page_of = tile + lane < t_end ? row_of_table[(tile + lane) >> page_shift] : -1;
    if (page_of >= a.c.n_pages) page_of = -1;
    const long at = (long)(page_of < 0 ? 0 : page_of) * a.c.n_kv + h;
    k_scale_of = a.c.k_scale[at];
    v_scale_of = a.c.v_scale[at];
  };
  auto lane_of = [](auto x, int tile) {
    return __builtin_bit_cast(decltype(x), __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), tile));
  };
  // The thread's chunks of a tile, and where they lie in LDS.  K: of 32 rows and 16 channels, [32 tokens][16 channels][half][row]; V: of 16
  // tokens and 32 channels, [16 tokens][32 channels][half][channel].  (Where there is no page, the first one's data, which no row sees.)
  u32x4_t kw[kChunks], vw[kChunks];
  auto from = [&](const uint8_t* base, int tile) {
    const int id = lane_of(page_of, tile - known);
    return reinterpret_cast<const u32x4_t*>(base + ((long)(id < 0 ? 0 : id) * a.c.n_kv + h) * a.c.page * D +
                                            (long)(id < 0 ? 0 : tile & page_mask) * kKvTile * D);
  };
  auto load_k = [&](int tile) {
    const u32x4_t* p = from(a.c.k, tile);
#pragma unroll
    for (int n = 0; n < kChunks; ++n) {
      const int u = (n * kAttnThreads + tid) >> 5, rr = tid & 31;       // u: (32 tokens, 16 channels)
      const int jr = rr & 3, hh = rr >> 2 & 1, jq = rr >> 3 & 1, sl = rr >> 4;
      kw[n] = p[((2 * hh + jq) * kKs + u % kKs) * 16 + 4 * (2 * (u / kKs) + sl) + jr];
    }
  };
  auto load_v = [&](int tile) {
    const u32x4_t* p = from(a.c.v, tile);
#pragma unroll
    for (int n = 0; n < kChunks; ++n) {
      const int u = (n * kAttnThreads + tid) >> 5, rr = tid & 31;       // u: (16 tokens u % 4, 32 channels)
      vw[n] = p[((2 * (u / 4) + (rr >> 4)) * 4 + u % 4) * 16 + (rr & 15)];
    }
  };
  auto store_k = [&](int buf, int n) {
    {
      f16x8_t* k = reinterpret_cast<f16x8_t*>(lds + buf * P::kBuf + ((n * kAttnThreads + tid) >> 5) * 1024) + (tid & 31);
      k[0] = attn_codes(kw[n][0], kw[n][1]);
      k[32] = attn_codes(kw[n][2], kw[n][3]);
    }
  };
  auto store_v = [&](int buf, int n) {
    {
      const int u = (n * kAttnThreads + tid) >> 5;
      f16x8_t* v = reinterpret_cast<f16x8_t*>(lds + (2 + buf) * P::kBuf + ((u % 4) * kDt + u / 4) * 1024) + (tid & 31);
      v[0] = attn_codes(vw[n][0], vw[n][1]);
      v[32] = attn_codes(vw[n][2], vw[n][3]);
    }
  };

  f32x16_t o[kDt];
#pragma unroll
  for (int d = 0; d < kDt; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  float m = -__builtin_huge_valf(), l = 0.f;             // reference and sum of the lane's row (half of its tokens)
  float mv = -__builtin_huge_valf();                     // reference of the row's sums of p v
  // Operands from LDS come kG at a time, a group ahead of their products; the barriers for the scheduler keep it so.
  constexpr int kG = kDt > 2 ? kDt / 2 : kDt, kGroups = 4 * kDt / kG;
  f16x8_t part[2][kG];
  auto read_k = [&](int buf, int g) {
#pragma unroll
    for (int n = 0; n < kG; ++n) part[g & 1][n] = *reinterpret_cast<const f16x8_t*>(lds + buf * P::kBuf + 16 * lane + (g * kG + n) * 1024);
  };
  auto read_v = [&](int buf, int g) {
#pragma unroll
    for (int n = 0; n < kG; ++n)
      part[g & 1][n] = *reinterpret_cast<const f16x8_t*>(lds + (2 + buf) * P::kBuf + 16 * lane + (g * kG + n) * 1024);
  };
  auto scores = [&](f32x16_t (&s)[2], int g) {           // of a group: products g kG .. of half u of the tokens, channels 16 k ..
#pragma unroll
    for (int n = 0; n < kG; ++n) {
      const int u = (g * kG + n) / kKs, k = (g * kG + n) % kKs;
      if (k == 0) s[u] = f32x16_t{};
      s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(part[g & 1][n], qf[k], s[u], 0, 0, 0);
    }
  };
  // Of a tile: its scores while the tile before goes through its softmax; K is two tiles ahead of the products with V, V one.
  f32x16_t s0[2], s1[2];
  if (t_begin < t_end) {
    learn(t_begin);
    load_k(t_begin);
    load_v(t_begin);
#pragma unroll
    for (int n = 0; n < kChunks; ++n) {
      store_k(0, n);
      store_v(0, n);
    }
    load_k(t_begin + 1);
    __syncthreads();
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      read_k(0, g);
      scores(s0, g);
    }
#pragma unroll
    for (int n = 0; n < kChunks; ++n) store_k(1, n);
    load_k(t_begin + 2);
    load_v(t_begin + 1);
    __syncthreads();
  }
  auto step = [&](int tile, f32x16_t (&s)[2], f32x16_t (&s_next)[2]) {
    const int buf = (tile - t_begin) & 1, t0 = tile * kKvTile;
    read_k(buf ^ 1, 0);
    if (tile + 3 > known + 63) learn(tile);
    const bool there = lane_of(page_of, tile - known) >= 0;
    const float k_scale = lane_of(k_scale_of, tile - known);
    const float v_scale = lane_of(v_scale_of, tile - known);
    const bool bad = !(k_scale < __builtin_huge_valf()) || !(v_scale < __builtin_huge_valf());
    const float log_v = bad ? 0.f : __builtin_amdgcn_logf(fmaxf(v_scale, 0x1p-120f));
    float f = k_scale * q_scale;
    // scores of register e of half u: token t0 + 32 u + 16 (e / 8) + 8 half + e % 8
    if (t0 < all_lo || t0 + kKvTile > all_hi || bad || !there) {        // uniform
      const int lo = see_lo - t0 - 8 * half, hi = there ? see_hi - t0 - 8 * half : lo;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int t = 32 * u + 16 * (e / 8) + e % 8;
          // a scale that is not finite reaches the rows that see the tile, and no others
          s[u][e] = t >= lo && t < hi ? bad ? __builtin_nanf("") : s[u][e] : -__builtin_huge_valf();
        }
      if (bad) f = 1.f;
    }
    f = fmaxf(f, 0x1p-126f);                             // what is hidden stays so under any scale
    float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(fmaxf(s[0][e], s[1][e]), top);
    top = fmaxf(top, __shfl_xor(top, 32, 64)) * f;
    const float top_v = top + log_v;
    if (__any(top > m + 8.f || top_v > mv + 8.f)) {
      const float m_new = fmaxf(m, top), mv_new = fmaxf(mv, top_v);
      const bool none = m_new == -__builtin_huge_valf(); // so far the row has seen nothing
      const float fade = none ? 1.f : __builtin_amdgcn_exp2f(m - m_new), fade_v = none ? 1.f : __builtin_amdgcn_exp2f(mv - mv_new);
      m = m_new;
      mv = mv_new;
      l *= fade;
#pragma unroll
      for (int d = 0; d < kDt; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= fade_v;
    }
    const bool none = m == -__builtin_huge_valf();
    const float base = none ? 0.f : fmaxf(log_v + (m - mv) + 7.f, -57.f) - m;
    __builtin_amdgcn_sched_barrier(0);

    // the next tile's scores beside this one's exponentials
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    f16x8_t p[4];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      if (g + 1 < kGroups) read_k(buf ^ 1, g + 1);
      else read_v(buf, 0);
      scores(s_next, g);
#pragma unroll
      for (int n = g * (32 / kGroups); n < (g + 1) * (32 / kGroups); ++n) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[n / 16][n % 16], f, base));
        sum[n & 3] += x;
        p[n / 8][n % 8] = (_Float16)x;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    const float undo = none ? 1.f : __builtin_amdgcn_exp2f(-(base + m));
    l = fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), undo, l);
    // K two tiles ahead and V one are made beside its products
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      if (g + 1 < kGroups) read_v(buf, g + 1);
#pragma unroll
      for (int n = 0; n < kG; ++n) {
        const int k = (g * kG + n) / kDt, d = (g * kG + n) % kDt;
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(part[g & 1][n], p[k], o[d], 0, 0, 0);
      }
      if (g % 2 == 0 && g < 2 * kChunks) store_k(buf, g / 2);
      if (g % 2 == 1 && g < 2 * kChunks) store_v(buf ^ 1, g / 2);
      __builtin_amdgcn_sched_barrier(0);
    }
    load_k(tile + 3);
    load_v(tile + 2);
    __syncthreads();
  };
  for (int tile = t_begin; tile < t_end; tile += 2) {
    step(tile, s0, s1);
    if (tile + 1 < t_end) step(tile + 1, s1, s0);
  }
  l += __shfl_xor(l, 32, 64);
  if (!on) return;
  // of the sums, to the units of l
  const float back = m == -__builtin_huge_valf() ? 1.f : __builtin_amdgcn_exp2f(mv - m - 7.f);
  // a block's channels 8 q + 4 half + j
  if (n_chunk > 1) {
    const long slot = (((long)seq * a.q_tiles + q_tile) * a.c.n_kv + h) * a.n_chunk + chunk;
    const long n_slot = (long)gridDim.y * a.q_tiles * a.c.n_kv * a.n_chunk;
    float* to = a.part + (slot * ROWS + r - it.r0) * D;
#pragma unroll
    for (int d = 0; d < kDt; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4_t*>(to + 32 * d + 8 * q + 4 * half) =
            f32x4_t{o[d][4 * q] * back, o[d][4 * q + 1] * back, o[d][4 * q + 2] * back, o[d][4 * q + 3] * back};
    if (half == 0) {
      float* ml = a.part + n_slot * ROWS * D + (slot * ROWS + r - it.r0) * 2;
      ml[0] = l == 0.f ? -__builtin_huge_valf() : m;
      ml[1] = l;
    }
  } else {
    T* to = static_cast<T*>(a.out) + (long)(it.first + i) * a.ldo + (long)head * D;
    const float f = l == 0.f ? 0.f : back / l;
#pragma unroll
    for (int d = 0; d < kDt; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        attn_store4(to + 32 * d + 8 * q + 4 * half, f32x4_t{o[d][4 * q], o[d][4 * q + 1], o[d][4 * q + 2], o[d][4 * q + 3]} * f, a.vec_o);
    if (a.lse && half == 0)
      a.lse[(long)(it.first + i) * a.n_q + head] = l == 0.f ? -__builtin_huge_valf() : (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

// Joins the chunks of a row.  One work-group per row: D / 4 threads hold four values of it each, and kParts such sets take every
// kParts-th chunk; their sums meet in LDS in order.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(kAttnThreads) void attn_join_kernel(AttnArgs a) {
  constexpr int kQuads = D / 4, kParts = kAttnThreads / kQuads;
  __shared__ f32x4_t sum_s[kParts][kQuads];
  __shared__ float weight_s[kAttnMostChunks], top_s[kAttnWaves], l_s[kAttnWaves];
  const int r = blockIdx.x % ROWS, item = blockIdx.x / ROWS;
  const int h = item % a.c.n_kv, q_tile = item / a.c.n_kv, seq = blockIdx.y;
  const AttnItem it = attn_item<ROWS>(a, seq, q_tile);
  if (!it.there || it.r0 + r >= it.rows) return;         // uniform
  const int n_chunk = attn_chunks(it, a.chunk_tiles);
  if (n_chunk <= 1) return;                              // written by the first launch
  const long slot = (((long)seq * a.q_tiles + q_tile) * a.c.n_kv + h) * a.n_chunk;
  const long n_slot = (long)gridDim.y * a.q_tiles * a.c.n_kv * a.n_chunk;
  const float* ml = a.part + n_slot * ROWS * D + (slot * ROWS + r) * 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float m[kAttnMostChunks / kAttnThreads], l[kAttnMostChunks / kAttnThreads], top = -__builtin_huge_valf();
#pragma unroll
  for (int k = 0; k < kAttnMostChunks / kAttnThreads; ++k) {
    const int c = k * kAttnThreads + tid;
    m[k] = c < n_chunk ? ml[(long)c * ROWS * 2] : -__builtin_huge_valf();
    l[k] = c < n_chunk ? ml[(long)c * ROWS * 2 + 1] : 0.f;
    top = fmaxf(top, m[k]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if (lane == 0) top_s[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kAttnWaves; ++w) top = fmaxf(top, top_s[w]);
  float total = 0.f;
#pragma unroll
  for (int k = 0; k < kAttnMostChunks / kAttnThreads; ++k) {
    const int c = k * kAttnThreads + tid;
    // a chunk that saw nothing has zero sums (or a NaN, which stays)
    const float f = m[k] == -__builtin_huge_valf() ? 1.f : __builtin_amdgcn_exp2f(m[k] - top);
    if (c < n_chunk) weight_s[c] = f;
    total += l[k] * f;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
  if (lane == 0) l_s[wave] = total;
  __syncthreads();
  total = 0.f;
#pragma unroll
  for (int w = 0; w < kAttnWaves; ++w) total += l_s[w];
  const int quad = tid % kQuads, first = tid / kQuads;
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  const float* from = a.part + (slot * ROWS + r) * D + 4 * quad;
#pragma unroll 4
  for (int c = first; c < n_chunk; c += kParts) {
    const f32x4_t part = *reinterpret_cast<const f32x4_t*>(from + (long)c * ROWS * D);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(part[e], weight_s[c], v[e]);
  }
  sum_s[first][quad] = v;
  __syncthreads();
  if (first > 0) return;
#pragma unroll
  for (int k = 1; k < kParts; ++k) v += sum_s[k][quad];
  const int i = (it.r0 + r) / a.group, head = h * a.group + (it.r0 + r) % a.group;
  T* to = static_cast<T*>(a.out) + (long)(it.first + i) * a.ldo + (long)head * D + 4 * quad;
  const float f = total == 0.f ? 0.f : 1.f / total;
  attn_store4(to, v * f, a.vec_o);
  if (a.lse && quad == 0)
    a.lse[(long)(it.first + i) * a.n_q + head] = total == 0.f ? -__builtin_huge_valf() : (top + __builtin_amdgcn_logf(total)) * kLn2;
}

// How a call is laid out: rows to a work item, work items along the queries, chunks along the cache.
constexpr int kAttnGroups = 1536, kAttnPromptGroups = 512;

struct AttnPlan {
  int rows, q_tiles, n_chunk, chunk_tiles;
  size_t ws_bytes;
};

// A window that reaches over every cache is none.
static int attn_window(int window, int max_kv) { return window < max_kv ? window : 0; }

static AttnPlan attn_plan(int n_seq, int max_q, int max_kv, int n_q, int n_kv, int dim, int window) {
  AttnPlan p;
  const long rows = (long)max_q * (n_q / n_kv);
  p.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 128;
  p.q_tiles = (int)((rows + p.rows - 1) / p.rows);
  // tiles that a work item can see
  window = attn_window(window, max_kv);
  long span = max_kv;
  if (window > 0 && window + (long)max_q < span) span = window + (long)max_q;
  const int tiles = (int)((span + kKvTile - 1) / kKvTile) + (window > 0 ? 1 : 0);
  // kAttnGroups work-groups; a chunk has at least a tile for each wavefront, or four where there are enough work items to begin with.
  // (Measured: 32 sequences of 1 to 16384 tokens, 8 key heads, 146 us with 1024 work-groups, 128 with 1536, 138 with 2048.)  Up to 16 tiles
  // the second launch and its workspace cost more than they save: 1000 tokens, 4 key heads 9.8 us of the GPU in two launches, 11.0 in
  // one, but 3.5 us less of the host; 1500 tokens 9.8 and 14.5.  (So a replayed graph, without the host, loses 1.2 us by it.)
  const long items = (long)n_seq * n_kv * p.q_tiles;
  const int least = items >= 256 ? 4 * kAttnWaves : kAttnWaves;
  long n = ((p.rows == 128 ? kAttnPromptGroups : kAttnGroups) + items - 1) / items;
  n = n < tiles / least ? n : tiles / least;
  n = n < kAttnMostChunks ? n : kAttnMostChunks;
  n = n > 1 && tiles > 16 ? n : 1;
  p.chunk_tiles = bpdq_ceil_div(bpdq_ceil_div(tiles > 0 ? tiles : 1, (int)n), kAttnWaves) * kAttnWaves;
  p.n_chunk = bpdq_ceil_div(tiles > 0 ? tiles : 1, p.chunk_tiles);
  p.ws_bytes = p.n_chunk > 1 ? (size_t)items * p.n_chunk * p.rows * (dim + 2) * sizeof(float) : 0;
  return p;
}

template <typename T, int D>
static int attn_launch(const AttnArgs& a, const AttnPlan& p, int n_seq, hipStream_t stream) {
  const dim3 grid((unsigned)(p.q_tiles * a.c.n_kv * p.n_chunk), n_seq);
  if (p.rows == 16) {
    hipLaunchKernelGGL((attn_rows_kernel<T, D, 1>), grid, dim3(kAttnThreads), 0, stream, a);
  } else if (p.rows == 32) {
    hipLaunchKernelGGL((attn_rows_kernel<T, D, 2>), grid, dim3(kAttnThreads), 0, stream, a);
  } else {
    BPDQ_HIP_TRY((bpdq_lds_limit<&attn_prompt_kernel<T, D>>(AttnPrompt<T, D>::kLds)));
    hipLaunchKernelGGL((attn_prompt_kernel<T, D>), grid, dim3(kAttnThreads), (AttnPrompt<T, D>::kLds), stream, a);
  }
  BPDQ_LAUNCH_CHECK();
  if (p.n_chunk > 1) {
    const dim3 join((unsigned)(p.q_tiles * a.c.n_kv * p.rows), n_seq);
    if (p.rows == 16) hipLaunchKernelGGL((attn_join_kernel<T, D, 16>), join, dim3(kAttnThreads), 0, stream, a);
    else if (p.rows == 32) hipLaunchKernelGGL((attn_join_kernel<T, D, 32>), join, dim3(kAttnThreads), 0, stream, a);
    else hipLaunchKernelGGL((attn_join_kernel<T, D, 128>), join, dim3(kAttnThreads), 0, stream, a);
    BPDQ_LAUNCH_CHECK();
  }
  return 0;
}

template <typename T>
static int attn_by_dim(const AttnArgs& a, const AttnPlan& p, int n_seq, hipStream_t stream) {
  switch (a.c.head_dim) {
    case 64: return attn_launch<T, 64>(a, p, n_seq, stream);
    case 128: return attn_launch<T, 128>(a, p, n_seq, stream);
    default: return attn_launch<T, 256>(a, p, n_seq, stream);
  }
}

}  // namespace bpdq

using namespace bpdq;

extern "C" size_t bpdq_kv_attention_workspace_bytes(int n_seq, int max_q, int max_kv, int n_q, int n_kv, int head_dim, int window) {
  if (n_seq <= 0 || max_q <= 0 || max_kv <= 0 || max_kv > kAttnMostKv || n_kv <= 0 || n_q <= 0 || n_q % n_kv || window < 0 ||
      (head_dim != 64 && head_dim != 128 && head_dim != 256) || (long)max_q * (n_q / n_kv) > (1L << 24))
    return 0;
  return attn_plan(n_seq, max_q, max_kv, n_q, n_kv, head_dim, window).ws_bytes;
}

extern "C" int bpdq_kv_attention(const bpdq_kv_cache* cache, const int* page_table, int max_pages, int n_seq, const int* kv_len,
                                 const int* q_start, int n_tok, int max_q, int max_kv, const void* Q, long ldq, int n_q,
                                 int dtype, float scale, int causal, int window, void* out, long ldo, float* lse, void* ws,
                                 size_t ws_bytes, void* stream_) {
  if (!kv_cache_ok(cache)) return -1;
  if (max_pages <= 0) return -3;
  if (n_seq < 0 || n_seq > 65535) return -4;
  if (n_tok < 0) return -7;
  if (n_q <= 0 || n_q % cache->n_kv) return -12;
  const int group = n_q / cache->n_kv;
  if (max_q < 0 || (long)max_q * group > (1L << 24)) return -8;
  if (max_kv < 0 || max_kv > kAttnMostKv || max_kv > (long)max_pages * cache->page) return -9;
  if (dtype != BPDQ_F16 && dtype != BPDQ_BF16) return -13;
  if (!(scale - scale == 0.f)) return -14;
  if (window < 0) return -16;
  if (n_seq == 0 || n_tok == 0 || max_q == 0) return 0;
  const long row = (long)n_q * cache->head_dim;
  if (!page_table) return -2;
  if (!kv_len) return -5;
  if (!q_start) return -6;
  if (!Q || (reinterpret_cast<uintptr_t>(Q) & 1)) return -10;
  if (ldq < row) return -11;
  if (!out || (reinterpret_cast<uintptr_t>(out) & 1)) return -17;
  if (ldo < row) return -18;
  const AttnPlan p = attn_plan(n_seq, max_q, max_kv, n_q, cache->n_kv, cache->head_dim, window);
  // threads along the grids' x
  if ((long)p.q_tiles * cache->n_kv * p.n_chunk * kAttnThreads > 0xffffffffL) return -8;
  if (p.n_chunk > 1 && (long)p.q_tiles * cache->n_kv * p.rows * kAttnThreads > 0xffffffffL) return -8;
  if (p.ws_bytes && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255))) return -20;
  if (ws_bytes < p.ws_bytes) return -21;
  AttnArgs a;
  a.c = *cache;
  a.table = page_table;
  a.kv_len = kv_len;
  a.q_start = q_start;
  a.q = Q;
  a.out = out;
  a.lse = lse;
  a.part = static_cast<float*>(ws);
  a.ldq = ldq;
  a.ldo = ldo;
  a.max_pages = max_pages;
  a.n_tok = n_tok;
  a.max_q = max_q;
  a.max_kv = max_kv;
  a.n_q = n_q;
  a.group = group;
  a.causal = causal != 0;
  a.vec_q = reinterpret_cast<uintptr_t>(Q) % 16 == 0 && ldq % 8 == 0;
  a.vec_o = reinterpret_cast<uintptr_t>(out) % 8 == 0 && ldo % 4 == 0;
  a.page_shift = cache->page == 64 ? 0 : cache->page == 128 ? 1 : 2;
  a.window = attn_window(window, max_kv);
  a.q_tiles = p.q_tiles;
  a.n_chunk = p.n_chunk;
  a.chunk_tiles = p.chunk_tiles;
  a.scale = scale;
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  return dtype == BPDQ_F16 ? attn_by_dim<_Float16>(a, p, n_seq, stream) : attn_by_dim<__bf16>(a, p, n_seq, stream);
}
