// Y = act(X What^T + bias) + residual from the stored bit-plane format (paper Eq. 1; Sec. 5 discusses serving).
// The weights become operands of the 16-bit matrix instructions in registers (planes.h); they are never written anywhere.
//
// Few tokens: what bounds it is the planes' way from memory (k / 8 bytes per weight) and the vector instructions that turn
// codes into values.  A work-group of eight wavefronts owns 16 R rows and NT tiles of 16 tokens; its wavefronts split the columns, 512 at
// a time: lane (row l % 16, quarter l / 16) loads 16 bytes of each plane, its quarter's 128 columns, and is the operand of that row
// for these columns, whatever the order in which they are contracted.  The partial sums meet in LDS, in the order of the
// wavefronts.
#pragma once
#include "planes.h"

namespace bpdq {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct LinearArgs {
  const uint32_t* planes;
  const _Float16* coefs;
  const void* x;
  const void* bias;
  const void* residual;
  void* y;
  long ldx, ldr, ldy;
  int d_out, d_in, group, n_tok, act;
  int vec_x, vec_w, vec_r, vec_y;                        // whether X, the planes, the residual and Y go by 16 bytes
};

template <typename T>
__device__ __forceinline__ f32x4_t mfma_16x16x32(u32x4_t a, u32x4_t b, f32x4_t c) {
  if constexpr (__is_same(T, _Float16))
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

__device__ __forceinline__ float linear_act(float v, int act) {
  switch (act) {
    case BPDQ_ACT_RELU: return v > 0.f ? v : (v == v ? 0.f : v);
    case BPDQ_ACT_GELU: return 0.5f * v * (1.f + erff(v * 0.70710678118654752440f));
    case BPDQ_ACT_GELU_TANH: {
      // 1 + tanh(u) = 2 / (1 + exp(-2u))
      const float u = 0.79788456080286535588f * (v + 0.044715f * v * v * v);
      return v / (1.f + __expf(-2.f * u));
    }
    case BPDQ_ACT_SILU: return v / (1.f + __expf(-v));
    default: return v;
  }
}

// 32 columns of a row of X, zeros from column d_in on (`columns` of them are there)
template <typename T>
__device__ __forceinline__ void linear_load_x(const T* __restrict__ x, int columns, bool vec, uint32_t (&out)[16]) {
  if (columns <= 0) {
#pragma unroll
    for (int q = 0; q < 16; ++q) out[q] = 0;
  } else if (vec) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const u32x4_t v = reinterpret_cast<const u32x4_t*>(x)[q];
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * q + e] = v[e];
    }
  } else {
    const unsigned short* s = reinterpret_cast<const unsigned short*>(x);
#pragma unroll
    for (int q = 0; q < 16; ++q) out[q] = (uint32_t)s[2 * q] | (uint32_t)s[2 * q + 1] << 16;
  }
}

// four consecutive words of a plane's row, of which `words` are there, the others zero
__device__ __forceinline__ u32x4_t linear_load_w(const uint32_t* __restrict__ p, int words, bool vec) {
  if (vec && words >= 4) return *reinterpret_cast<const u32x4_t*>(p);
  u32x4_t w = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < words) w[j] = p[j];
  return w;
}

constexpr int kLinThreads = 512;
constexpr int kLinWaves = kLinThreads / 64;

template <typename T, int K, int R, int NT>
__global__ __launch_bounds__(kLinThreads) void linear_rows_kernel(LinearArgs a) {
  constexpr int kRows = 16 * R, kToks = 16 * NT;
  __shared__ float part[kLinWaves][kToks][kRows];
  const int tid = threadIdx.x, lane = tid & 63, low = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = blockIdx.x * kRows, tok0 = blockIdx.y * kToks;
  const int nw = a.d_in / 32, n_grp = a.d_in / a.group, wpg = a.group / 32;

  f32x4_t acc[R][NT];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[r][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  long row[R];
  const T* x[NT];
#pragma unroll
  for (int r = 0; r < R; ++r) row[r] = row0 + 16 * r + low < a.d_out ? row0 + 16 * r + low : a.d_out - 1;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int t = tok0 + 16 * n + low;
    x[n] = static_cast<const T*>(a.x) + (t < a.n_tok ? t : a.n_tok - 1) * a.ldx;
  }
  for (int w0 = 16 * wave; w0 < nw; w0 += 16 * kLinWaves) {
    const int word = w0 + 4 * quarter;                   // the lane's words: word .. word + 3
    const int there = nw - word;
    u32x4_t w[R][K];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < K; ++i)
        w[r][i] = linear_load_w(a.planes + ((long)i * a.d_out + row[r]) * nw + (there > 0 ? word : 0), there, a.vec_w);
    PlaneLevels<T, K> levels[R];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool on = j < there;
      // a group's first word, or the lane's first (which may lie inside a group)
      if (j == 0 || wpg % 4 != 0) {
        const int grp = (on ? word + j : 0) / wpg;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          _Float16 c[K + 1];
#pragma unroll
          for (int i = 0; i <= K; ++i) {
            c[i] = a.coefs[((long)i * a.d_out + row[r]) * n_grp + grp];
            if (!on) c[i] = (_Float16)0.f;               // words past the end add nothing
          }
          levels[r].set(c);
        }
      }
      u32x4_t xs[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        uint32_t raw[16];
        linear_load_x(x[n] + 32L * (on ? word + j : 0), on ? 32 : 0, a.vec_x, raw);
        plane_order(raw, xs[n]);
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        uint32_t words[K];
#pragma unroll
        for (int i = 0; i < K; ++i) words[i] = w[r][i][j];
        const PlaneWord<K> pw(words);
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const u32x4_t v = pw.template values<T, false>(levels[r], f);
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[r][n] = mfma_16x16x32<T>(v, xs[n][f], acc[r][n]);
        }
      }
    }
  }
  // acc: row 4 quarter + i of the tile, token low
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
      *reinterpret_cast<f32x4_t*>(&part[wave][16 * n + low][16 * r + 4 * quarter]) = acc[r][n];
  __syncthreads();
  for (int id = tid; id < kRows * kToks; id += kLinThreads) {
    const int r = row0 + id % kRows, t = tok0 + id / kRows;
    if (r >= a.d_out || t >= a.n_tok) continue;
    float v = 0.f;
#pragma unroll
    for (int s = 0; s < kLinWaves; ++s) v += part[s][id / kRows][id % kRows];
    if (a.bias) v += (float)static_cast<const T*>(a.bias)[r];
    v = linear_act(v, a.act);
    if (a.residual) v += (float)static_cast<const T*>(a.residual)[t * a.ldr + r];
    static_cast<T*>(a.y)[t * a.ldy + r] = (T)v;
  }
}

template <typename T>
__device__ __forceinline__ f32x16_t mfma_32x32x16(u32x4_t a, u32x4_t b, f32x16_t c) {
  if constexpr (__is_same(T, _Float16))
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Shape of a work-group of the tile kernel: WR x WT wavefronts of RT x TT blocks of 32 rows x 32 tokens, KS times over the columns.
template <int K, int WR_, int WT_, int KS_, int RT_, int TT_>
struct LinearTile {
  static constexpr int WR = WR_, WT = WT_, KS = KS_, RT = RT_, TT = TT_;
  static constexpr int kRows = 32 * RT * WR, kToks = 32 * TT * WT;
  static constexpr int kPart = 64 * WR * WT, kThreads = kPart * KS;
  static constexpr int kWords = K <= 2 ? 4 : 2;          // consecutive words of a lane: fewer where more planes take the registers
  static constexpr int kPieces = kToks * 8 / kPart;      // 16-byte pieces of X that a thread moves per 64 columns
  static constexpr int kBuf = kToks * 128;               // bytes of 64 columns of X
  static constexpr size_t kLds = (size_t)2 * KS * kBuf;
  static_assert(KS == 1 || (size_t)(KS / 2) * kRows * kToks * 4 <= kLds, "the joining of the parts has to fit");
};

// Eight rows from `first` of one token: bias, activation, residual, one rounding.
template <typename T>
__device__ __forceinline__ void linear_finish8(const LinearArgs& a, long tok, int first, f32x4_t v0, f32x4_t v1, bool vec_y,
                                               bool vec_r) {
  typedef T T8 __attribute__((ext_vector_type(8)));
  float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
  const int n = a.d_out - first < 8 ? a.d_out - first : 8;
  if (a.bias) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) v[i] += (float)static_cast<const T*>(a.bias)[first + i];
  }
  if (a.act != BPDQ_ACT_NONE) {
#pragma unroll 1
    for (int i = 0; i < 8; i += 2) {                     // (indexed by registers below: two at a time keep the code small)
      const float p = linear_act(i == 0 ? v[0] : i == 2 ? v[2] : i == 4 ? v[4] : v[6], a.act);
      const float q = linear_act(i == 0 ? v[1] : i == 2 ? v[3] : i == 4 ? v[5] : v[7], a.act);
      if (i == 0) { v[0] = p; v[1] = q; }
      else if (i == 2) { v[2] = p; v[3] = q; }
      else if (i == 4) { v[4] = p; v[5] = q; }
      else { v[6] = p; v[7] = q; }
    }
  }
  if (a.residual) {
    const T* r = static_cast<const T*>(a.residual) + tok * a.ldr + first;
    if (vec_r && n == 8) {
      const T8 add = *reinterpret_cast<const T8*>(r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += (float)add[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) v[i] += (float)r[i];
    }
  }
  T* y = static_cast<T*>(a.y) + tok * a.ldy + first;
  if (vec_y && n == 8) {
    T8 out;
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = (T)v[i];
    *reinterpret_cast<T8*>(y) = out;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) y[i] = (T)v[i];
  }
}

template <typename T, int K, typename S>
__global__ __launch_bounds__(S::kThreads) void linear_tiles_kernel(LinearArgs a, int tok_tiles) {
  constexpr int W = S::kWords, RT = S::RT, TT = S::TT;
  extern __shared__ uint4 lds_raw[];
  char* lds = reinterpret_cast<char*>(lds_raw);
  const int part = __builtin_amdgcn_readfirstlane(threadIdx.x / S::kPart);
  const int tid = threadIdx.x % S::kPart, lane = tid & 63, low = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % S::WR, wt = wave / S::WR;
  const int row0 = blockIdx.x / tok_tiles * S::kRows, tok0 = blockIdx.x % tok_tiles * S::kToks;
  const int nw = a.d_in / 32, n_grp = a.d_in / a.group, wpg = a.group / 32;
  const int grp_step = wpg % 4 == 0 ? 4 : wpg % 2 == 0 ? 2 : 1;     // words after which a lane's group may change

  // where the thread's pieces of X and the lane's rows lie, as byte offsets from the tile's first token and row
  const char* x_base = reinterpret_cast<const char*>(a.x) + (long)tok0 * a.ldx * 2;
  const int piece = tid & 3, unit0 = tid >> 2;           // unit: (token, half)
  const int x_tok = unit0 >> 1, x_half = unit0 & 1, x_last = a.n_tok - 1 - tok0;
  const unsigned x_row = (unsigned)a.ldx * 2u;
  constexpr int kTokStep = S::kPart / 8;                 // tokens between a thread's pieces
  static_assert(kTokStep % 8 == 0, "a thread's pieces lie alike in LDS");
  const unsigned x_lds = (unsigned)(x_tok * 128 + ((4 * x_half) ^ (x_tok & 7)) * 16 + piece * 4);
  const char* w_base[K];
  const char* c_base[K + 1];
#pragma unroll
  for (int i = 0; i < K; ++i) w_base[i] = reinterpret_cast<const char*>(a.planes + ((long)i * a.d_out + row0) * nw);
#pragma unroll
  for (int i = 0; i <= K; ++i) c_base[i] = reinterpret_cast<const char*>(a.coefs + ((long)i * a.d_out + row0) * n_grp);
  unsigned row[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int at = 32 * (RT * wr + r) + low;
    row[r] = row0 + at < a.d_out ? at : a.d_out - 1 - row0;
  }

  u32x4_t xv[S::kPieces];
  auto load_x = [&](int chunk, int j) {                  // sub-chunk j: word j of each half
    const int word = 2 * W * chunk + W * x_half + j;
    const bool on = word < nw;
    const unsigned col = (unsigned)(on ? word : 0) * 64u + (unsigned)piece * 16u;
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) {
      const int t = x_tok + i * kTokStep < x_last ? x_tok + i * kTokStep : x_last;
      const char* p = x_base + ((unsigned)t * x_row + col);
      u32x4_t v;
      if (a.vec_x) {
        v = *reinterpret_cast<const u32x4_t*>(p);
      } else {
        const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (uint32_t)s[2 * e] | (uint32_t)s[2 * e + 1] << 16;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) xv[i][e] = on ? v[e] : 0u;
    }
  };
  auto store_x = [&](int buf) {
    char* at = lds + (part * 2 + buf) * S::kBuf;
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i)
#pragma unroll
      for (int f = 0; f < 4; ++f)                        // (4 h + f) ^ (t & 7): f changes the two lowest bits of the slot
        *reinterpret_cast<uint32_t*>(at + (x_lds ^ (unsigned)(f * 16)) + i * (kTokStep * 128)) = xv[i][f];
  };
  uint32_t w_cur[RT][K][W], w_next[RT][K][W];
  auto load_w = [&](int chunk, uint32_t (&w)[RT][K][W]) {
    const int word = 2 * W * chunk + W * half;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const char* p = w_base[i] + (row[r] * (unsigned)nw + (unsigned)(word < nw ? word : 0)) * 4u;
        if (a.vec_w) {                                   // rows of whole lanes
          typedef uint32_t words __attribute__((ext_vector_type(W)));
          const words v = *reinterpret_cast<const words*>(p);
#pragma unroll
          for (int j = 0; j < W; ++j) w[r][i][j] = v[j];
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j) w[r][i][j] = word + j < nw ? reinterpret_cast<const uint32_t*>(p)[j] : 0u;
        }
      }
  };
  _Float16 c_next[RT][K + 1];
  auto load_c = [&](int chunk, int j) {
    const int word = 2 * W * chunk + W * half + j;
    const unsigned g = (unsigned)(word < nw ? word : 0) / (unsigned)wpg;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i <= K; ++i) {
        const _Float16 v = *reinterpret_cast<const _Float16*>(c_base[i] + (row[r] * (unsigned)n_grp + g) * 2u);
        c_next[r][i] = word < nw ? v : (_Float16)0.f;    // words past the end add nothing
      }
  };

  f32x16_t acc[RT][TT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[r][t][e] = 0.f;
  PlaneLevels<T, K> levels[RT];

  const int n_chunk = bpdq_ceil_div(nw, 2 * W * S::KS);  // chunks of a part, the last ones maybe empty
  load_x(part, 0);
  load_w(part, w_next);
  load_c(part, 0);
  store_x(0);
  load_x(part, 1);
  __syncthreads();
  for (int n = 0; n < n_chunk; ++n) {
    const int chunk = n * S::KS + part, chunk1 = chunk + S::KS;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < K; ++i)
#pragma unroll
        for (int j = 0; j < W; ++j) w_cur[r][i][j] = w_next[r][i][j];
    load_w(chunk1, w_next);
#pragma unroll
    for (int j = 0; j < W; ++j) {
      store_x((j + 1) & 1);
      load_x(j + 2 < W ? chunk : chunk1, (j + 2) % W);
      if (j % grp_step == 0) {
#pragma unroll
        for (int r = 0; r < RT; ++r) levels[r].set(c_next[r]);
        if (j + grp_step < W) load_c(chunk, j + grp_step);
        else load_c(chunk1, 0);
      }
      const char* at = lds + (part * 2 + (j & 1)) * S::kBuf;
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        u32x4_t b[TT];
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          const int tok = 32 * (TT * wt + t) + low;
          b[t] = *reinterpret_cast<const u32x4_t*>(at + tok * 128 + (((4 * half + f) ^ (tok & 7)) * 16));
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          uint32_t words[K];
#pragma unroll
          for (int i = 0; i < K; ++i) words[i] = w_cur[r][i][j];
          const u32x4_t v = PlaneWord<K>(words).template values<T, true>(levels[r], f);
#pragma unroll
          for (int t = 0; t < TT; ++t) acc[r][t] = mfma_32x32x16<T>(v, b[t], acc[r][t]);
        }
      }
      __syncthreads();
    }
  }

  // the parts' sums meet in LDS, the upper half of the parts added to the lower until one is left
  if constexpr (S::KS > 1) {
    float* sum = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int left = S::KS / 2; left > 0; left /= 2) {
      if (part >= left && part < 2 * left) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              sum[((((part - left) * S::WR * S::WT + wave) * RT + r) * TT + t) * 1024 + e * 64 + lane] = acc[r][t][e];
      }
      __syncthreads();
      if (part < left) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              acc[r][t][e] += sum[(((part * S::WR * S::WT + wave) * RT + r) * TT + t) * 1024 + e * 64 + lane];
      }
      __syncthreads();
    }
    if (part > 0) return;
  }
  // 32 tokens at a time through the wavefront's 8 KB of LDS, so that eight lanes store 128 consecutive bytes of a token; of a block a
  // lane holds rows 8 q + 4 half + i of token low.  (16-byte slot n of a token's 64 rows lies at n ^ (token & 15).)
  constexpr int kSlots = 8 * RT;
  static_assert(RT == 2 && (size_t)S::WR * S::WT * 32 * 64 * 4 <= S::kLds, "16 slots a token");
  f32x4_t* mine = reinterpret_cast<f32x4_t*>(lds) + wave * 32 * kSlots;
  const bool vec_y = a.vec_y, vec_r = a.vec_r;
#pragma unroll 1
  for (int t = 0; t < TT; ++t) {
#pragma unroll
    for (int u = 0; u < TT; ++u) {
      if (u != t) continue;                              // uniform: acc stays in registers
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          mine[low * kSlots + ((8 * r + 2 * q + half) ^ (low & 15))] =
              f32x4_t{acc[r][u][4 * q], acc[r][u][4 * q + 1], acc[r][u][4 * q + 2], acc[r][u][4 * q + 3]};
    }
    __builtin_amdgcn_wave_barrier();                     // (LDS serves a wavefront in order)
#pragma unroll 1
    for (int it = 0; it < 32 * kSlots / 2 / 64; ++it) {
      const int k = it * 8 + (lane >> 3), s2 = 2 * (lane & 7);
      const f32x4_t v0 = mine[k * kSlots + (s2 ^ (k & 15))], v1 = mine[k * kSlots + ((s2 + 1) ^ (k & 15))];
      const long tok = tok0 + 32 * (TT * wt + t) + k;
      const int first = row0 + 32 * RT * wr + 4 * s2;
      if (tok < a.n_tok && first < a.d_out) linear_finish8<T>(a, tok, first, v0, v1, vec_y, vec_r);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T, int K, typename S>
static int linear_launch_tiles(const LinearArgs& a, hipStream_t stream) {
  BPDQ_HIP_TRY((bpdq_lds_limit<&linear_tiles_kernel<T, K, S>>(S::kLds)));
  const int tok_tiles = bpdq_ceil_div(a.n_tok, S::kToks);
  hipLaunchKernelGGL((linear_tiles_kernel<T, K, S>), dim3(bpdq_ceil_div(a.d_out, S::kRows) * tok_tiles), dim3(S::kThreads), S::kLds,
                     stream, a, tok_tiles);
  BPDQ_LAUNCH_CHECK();
  return 0;
}

template <typename T, int K, int R, int NT>
static int linear_launch(const LinearArgs& a, hipStream_t stream) {
  const dim3 grid(bpdq_ceil_div(a.d_out, 16 * R), bpdq_ceil_div(a.n_tok, 16 * NT));
  hipLaunchKernelGGL((linear_rows_kernel<T, K, R, NT>), grid, dim3(kLinThreads), 0, stream, a);
  BPDQ_LAUNCH_CHECK();
  return 0;
}

template <typename T, int K>
static int linear_pick(const LinearArgs& a, hipStream_t stream) {
  if (a.n_tok <= 16) return linear_launch<T, K, 1, 1>(a, stream);
  // offsets inside a tile of X are 32 bits
  if (a.n_tok <= 32 || a.ldx >= 1L << 22) return linear_launch<T, K, 2, 2>(a, stream);
  if (a.n_tok <= 1024) return linear_launch_tiles<T, K, LinearTile<K, 2, 1, 4, 2, 4>>(a, stream);
  return linear_launch_tiles<T, K, LinearTile<K, 4, 2, 1, 2, 4>>(a, stream);
}

template <int K>
int linear_run(const LinearArgs& a, int dtype, hipStream_t stream) {
  return dtype == BPDQ_F16 ? linear_pick<_Float16, K>(a, stream) : linear_pick<__bf16, K>(a, stream);
}

// instantiated in linear_k1.hip to linear_k4.hip
extern template int linear_run<1>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<2>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<3>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<4>(const LinearArgs&, int, hipStream_t);

}  // namespace bpdq
