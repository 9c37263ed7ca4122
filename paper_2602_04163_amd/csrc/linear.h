// Y = act(X What^T + bias) + residual from the stored bit-plane format (paper Eq. 1; Sec. 5 discusses serving).
// The weights become operands of the 16-bit matrix instructions in registers (planes.h); they are never written anywhere.
//
// Few tokens: what bounds it is latency, beside the vector instructions that turn codes into values.  A work-group of eight
// wavefronts owns 16 R rows and NT tiles of 16 tokens; its wavefronts split the columns, 256 at a time: lane (row l % 16,
// quarter l / 16) loads 8 bytes of each plane, its quarter's 64 columns, and is the operand of that row for these columns,
// whatever the order in which they are contracted.  The partial sums meet in LDS, in the order of the wavefronts.
// One bf16 token, 3584 x 3584 at 2 bits in groups of 128: 7.0 to 7.2 us (3.8 MB; one round of 224 work-groups; a pass over the token for its
// power of two comes first).  16 fp16 tokens, 18944 x 3584 at 3 bits: 15 to 17 us for 30 MB, 1.8 to 2.0 TB/s: vector instructions issue in 55 % of the
// cycles, matrix instructions in 7 %; two wavefronts to a SIMD, X not requested ahead, and 14 rounds of columns dealt to eight
// wavefronts leave the rest empty.
//
// More tokens: tiles (linear_tiles_kernel), which decode a row's weights once for 64 to 256 tokens.
#pragma once
#include "linear_plan.h"
#include "planes.h"

#include <type_traits>

namespace bpdq {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

constexpr int kLinTokPad = 256;                           // the ordering covers whole tiles of any shape

static inline size_t linear_image_bytes(int n_tok, int d_in) {         // with an image of zeros to a block of 32 tokens
  return bpdq_align_up((size_t)n_tok, kLinTokPad) * (bpdq_align_up((size_t)d_in, 256) * 2 + 128);
}

struct LinearArgs {
  const uint32_t* planes;
  const _Float16* coefs;
  const void* x;
  const void* bias;
  const void* residual;
  void* y;
  void* ws;                                              // X in the order of the tile kernel
  long ldx, ldr, ldy;
  int d_out, d_in, group, n_tok, act;
  int vec_x, vec_w, vec_r, vec_y;                        // whether X, the planes, the residual and Y go by 16 bytes
};

__device__ __forceinline__ f32x4_t mfma_16x16x32(u32x4_t a, u32x4_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// X in bf16 as fp16.  Weights rounded to bf16 would cost as much accuracy again as the rounding of the result (measured: 1.4 to 1.6 times
// the error); fp16 has the bits of both, and a power of two per token brings its values into range, exactly but for those below 2^-29 of the token's
// largest.  The largest magnitude's exponent goes to that of [2^15, 2^16), on the bit patterns: pattern - base, in units of an
// exponent, saturating at zero, and three bits up.  (A row with an infinity or NaN keeps these.)
__device__ __forceinline__ uint32_t linear_base(uint32_t most) {        // of the token's largest pattern without sign
  const int e = most >> 7;
  return e == 255 ? 224u << 7 : e > 30 ? (uint32_t)(e - 30) << 7 : 0u;
}
__device__ __forceinline__ float linear_unscale(uint32_t base) { return ldexpf(1.f, (int)(base >> 7) - 112); }
__device__ __forceinline__ uint32_t linear_half2(uint32_t x, uint32_t base2) {       // base2: base in both halves
  typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
  const u16x2_t m = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2_t, x & 0x7fff7fffu), __builtin_bit_cast(u16x2_t, base2));
  return __builtin_bit_cast(uint32_t, m) << 3 | (x & 0x80008000u);
}
// the larger of the eight patterns without sign and of `most`
__device__ __forceinline__ uint32_t linear_most(u32x4_t v, uint32_t most) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t a = v[q] & 0x7fffu, b = v[q] >> 16 & 0x7fffu;
    most = most > a ? most : a;
    most = most > b ? most : b;
  }
  return most;
}
// GATED: the rows are those of two projections, gate and then up, of `half` rows each, and a tile takes them by eights in turn, so that
// the eight of a gate and the eight of its up meet in one wavefront's epilogue.  The stored row of a tile's row v (past the end: the last):
__device__ __forceinline__ int linear_pair_row(int v, int half) {
  const int f = (v >> 4) * 8 + (v & 7);
  return (f < half ? f : half - 1) + (v & 8 ? half : 0);
}
// eight consecutive values of X
template <typename T>
__device__ __forceinline__ u32x4_t linear_load8(const T* __restrict__ x, bool vec) {
  if (vec) return *reinterpret_cast<const u32x4_t*>(x);
  const unsigned short* s = reinterpret_cast<const unsigned short*>(x);
  u32x4_t v;
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = (uint32_t)s[2 * q] | (uint32_t)s[2 * q + 1] << 16;
  return v;
}

template <int ACT>
__device__ __forceinline__ float linear_act(float v) {
  if constexpr (ACT == BPDQ_ACT_RELU) return v > 0.f ? v : (v == v ? 0.f : v);
  if constexpr (ACT == BPDQ_ACT_GELU) {
    // v Phi(v): Phi(v) = erfc(-v / sqrt 2) / 2 below zero and 1 - erfc(v / sqrt 2) / 2 above, erfc(x) = exp(-x^2) P(t), t = 1 / (1 + 3/8 x), for
    // x >= 0.  P, of degree 7 without a constant, was fitted to exp(x^2) erfc(x) by the least largest relative error (9.2e-7 up to x = 12), so the
    // result is good to 5e-6 of itself wherever it is above fp32's denormals: a form with a small absolute error of erfc alone
    // loses half an fp16 step at v = -4, 1.5 % of the value at -9.
    const float t = __builtin_amdgcn_rcpf(fmaf(0.375f * 0.70710678118654752440f, fabsf(v), 1.f));
    float poly = fmaf(t, -0.13322853f, 0.38146659f);
    poly = fmaf(t, poly, -0.12063710f);
    poly = fmaf(t, poly, 0.27674545f);
    poly = fmaf(t, poly, 0.16904420f);
    poly = fmaf(t, poly, 0.21523673f);
    poly = fmaf(t, poly, 0.21137326f);
    const float tail = 0.5f * t * poly * __expf(-0.5f * v * v);
    return v * (v < 0.f ? tail : 1.f - tail);
  }
  if constexpr (ACT == BPDQ_ACT_GELU_TANH) {
    // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2u))
    const float u = 0.79788456080286535588f * (v + 0.044715f * v * v * v);
    return v * __builtin_amdgcn_rcpf(1.f + __expf(-2.f * u));
  }
  if constexpr (ACT == BPDQ_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.f + __expf(-v));
  return v;
}
__device__ __forceinline__ float linear_act(float v, int act) {
  switch (act) {
    case BPDQ_ACT_RELU: return linear_act<BPDQ_ACT_RELU>(v);
    case BPDQ_ACT_GELU: return linear_act<BPDQ_ACT_GELU>(v);
    case BPDQ_ACT_GELU_TANH: return linear_act<BPDQ_ACT_GELU_TANH>(v);
    case BPDQ_ACT_SILU: return linear_act<BPDQ_ACT_SILU>(v);
    default: return v;
  }
}

constexpr int kWords = 4;                                 // consecutive words of a lane in the tile kernel
constexpr int kLinThreads = 512;
constexpr int kLinWaves = kLinThreads / 64;

constexpr int kRowPitch = 512 + 16;                       // bytes of a token's 256 columns in LDS: 16 tokens fall into all 64 banks

// (Registers for one work-group to a CU: with the 128 of two, 16 rows spill, and 20 fp16 tokens of 11264 columns at 4 bits take 33 us, not 17.
// With all 256 the forms of one row tile have none in scratch; of the others 14 do, 6 to 74 registers: twice 16 tokens with five row tiles but for
// fp16 at one plane, with three at three and four planes, with two in bf16 at four, and eight row tiles at four.)
template <typename T, int K, int R, int NT, bool GATED>
__global__ __launch_bounds__(kLinThreads, 2) void linear_rows_kernel(LinearArgs a) {
  constexpr int kRows = 16 * R, kToks = 16 * NT;
  constexpr int kStageBytes = kLinWaves * 16 * kRowPitch, kPartBytes = kLinWaves * kToks * kRows * 4;
  __shared__ uint4 lds_raw[(kStageBytes > kPartBytes ? kStageBytes : kPartBytes) / 16];
  const int tid = threadIdx.x, lane = tid & 63, low = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = blockIdx.x * kRows, tok0 = blockIdx.y * kToks;
  const int nw = a.d_in / 32, n_grp = a.d_in / a.group, wpg = a.group / 32;
  const int toks = a.n_tok - tok0 < kToks ? a.n_tok - tok0 : kToks;
  char* stage = reinterpret_cast<char*>(lds_raw) + wave * 16 * kRowPitch;
  constexpr bool kScale = !__is_same(T, _Float16);
  __shared__ uint32_t most_s[kToks > kLinWaves ? kToks : kLinWaves], base_s[kToks];

  f32x4_t acc[R][NT];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[r][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // the next row tile's words and first coefficients, requested a tile ahead
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  u32x2_t w_next[K];
  _Float16 c_next[K + 1], c_next2[K + 1];                // of the first word and, where groups have an odd number of words, the second
  const bool odd = wpg % 2 != 0;
  auto row = [&](int r) { return GATED ? linear_pair_row(row0 + 16 * r + low, a.d_out / 2)
                                       : row0 + 16 * r + low < a.d_out ? row0 + 16 * r + low : a.d_out - 1; };
  auto load_c = [&](int r, int word, _Float16 (&c)[K + 1]) {
    const _Float16* p = a.coefs + (long)row(r) * n_grp + (word < nw ? word : 0) / wpg;
#pragma unroll
    for (int i = 0; i <= K; ++i) c[i] = p[(long)i * a.d_out * n_grp];
  };
  auto load_w = [&](int r, int word) {                   // words past the end: the row's first, under levels of zero
    const uint32_t* p = a.planes + (long)row(r) * nw;
#pragma unroll
    for (int i = 0; i < K; ++i, p += (long)a.d_out * nw) {
      if (a.vec_w) {
        w_next[i] = *reinterpret_cast<const u32x2_t*>(p + (word < nw ? word : 0));
      } else {
        w_next[i][0] = p[word < nw ? word : 0];
        w_next[i][1] = p[word + 1 < nw ? word + 1 : 0];
      }
    }
    load_c(r, word, c_next);
    if (odd) load_c(r, word + 1, c_next2);
  };
  if (8 * wave < nw) load_w(0, 8 * wave + 2 * quarter);
  if constexpr (kScale) {                                // (while the first words are on their way)
    // a power of two of threads to each token, so that all tokens are read at once
    const int share = 9 - (toks > 1 ? 32 - __builtin_clz(toks - 1) : 0), t = tid >> share;      // as powers of two
    const int lanes = 1 << share, part = share < 6 ? share : 6;
    uint32_t most = 0;
    if (t < toks) {
      const T* x = static_cast<const T*>(a.x) + (tok0 + t) * a.ldx;
#pragma unroll 4
      for (int c = 8 * (tid & (lanes - 1)); c < a.d_in; c += 8 * lanes) most = linear_most(linear_load8(x + c, a.vec_x), most);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      if (o >> part) continue;                           // uniform
      const uint32_t b = __shfl_xor(most, o, 64);
      most = most > b ? most : b;
    }
    if ((tid & ((1 << part) - 1)) == 0) most_s[tid >> part] = most;
    __syncthreads();
    if (tid < toks) {
      const int n = lanes >> part;
      uint32_t all = 0;
      for (int w = 0; w < n; ++w) all = all > most_s[tid * n + w] ? all : most_s[tid * n + w];
      base_s[tid] = linear_base(all);
    }
    __syncthreads();
  }
  for (int w0 = 8 * wave; w0 < nw; w0 += 8 * kLinWaves) {
    const int word = w0 + 2 * quarter;                   // the lane's words: word, word + 1
    // X of 256 columns to operands, 16 tokens at a time by way of LDS: loads of whole lines.  Rows behind the last token keep what LDS
    // held: their results are dropped.
    const int at = w0 + (lane >> 2 & 7);                 // word of the lane's 16 bytes
    u32x4_t xs[NT][2][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      u32x4_t v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (16 * n + 2 * i >= toks) break;               // uniform
        const int t = 16 * n + 2 * i + (lane >> 5) < toks ? 16 * n + 2 * i + (lane >> 5) : toks - 1;
        v[i] = linear_load8(static_cast<const T*>(a.x) + (tok0 + t) * a.ldx + (at < nw ? 8L * (4 * w0 + (lane & 31)) : 0L), a.vec_x);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (16 * n + 2 * i >= toks) break;
        if (at >= nw) v[i] = u32x4_t{0, 0, 0, 0};
        if constexpr (kScale) {
          const uint32_t base = base_s[16 * n + 2 * i + (lane >> 5) < toks ? 16 * n + 2 * i + (lane >> 5) : toks - 1] * 0x10001u;
#pragma unroll
          for (int q = 0; q < 4; ++q) v[i][q] = linear_half2(v[i][q], base);
        }
        *reinterpret_cast<u32x4_t*>(stage + (2 * i + (lane >> 5)) * kRowPitch + 16 * (lane & 31)) = v[i];
      }
      __builtin_amdgcn_wave_barrier();                   // (LDS serves a wavefront in order)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t raw[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const u32x4_t u = *reinterpret_cast<const u32x4_t*>(stage + low * kRowPitch + 128 * quarter + 64 * j + 16 * q);
#pragma unroll
          for (int e = 0; e < 4; ++e) raw[4 * q + e] = u[e];
        }
        plane_order(raw, xs[n][j]);
      }
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      u32x2_t w[K];
      _Float16 c[K + 1];
#pragma unroll
      for (int i = 0; i < K; ++i) w[i] = w_next[i];
#pragma unroll
      for (int i = 0; i <= K; ++i) c[i] = word < nw ? c_next[i] : (_Float16)0.f;      // words past the end add nothing
      _Float16 c2[K + 1];
#pragma unroll
      for (int i = 0; i <= K; ++i) c2[i] = word + 1 < nw && odd ? c_next2[i] : (_Float16)0.f;
      if (r + 1 < R) load_w(r + 1, word);
      else if (w0 + 8 * kLinWaves < nw) load_w(0, word + 8 * kLinWaves);
      PlaneLevels<K> levels;
      levels.set(c);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (j == 1 && odd) levels.set(c2);               // uniform: the second word may be another group's
        uint32_t words[K];
#pragma unroll
        for (int i = 0; i < K; ++i) words[i] = w[i][j];
        const PlaneWord<K> pw(words);
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const u32x4_t v = pw.values(levels, f);
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[r][n] = mfma_16x16x32(v, xs[n][j][f], acc[r][n]);
        }
      }
    }
  }
  __syncthreads();
  // acc: row 4 quarter + i of the tile, token low
  float* part = reinterpret_cast<float*>(lds_raw);       // [wave][token][row]
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
      *reinterpret_cast<f32x4_t*>(part + (wave * kToks + 16 * n + low) * kRows + 16 * r + 4 * quarter) = acc[r][n];
  __syncthreads();
  if constexpr (GATED) {
    const int f_all = a.d_out / 2;
    for (int id = tid; id < kRows / 2 * kToks; id += kLinThreads) {
      const int at = id % (kRows / 2), f = row0 / 2 + at, n = id / (kRows / 2), t = tok0 + n;
      if (f >= f_all || t >= a.n_tok) continue;
      const float* sum = part + n * kRows + 16 * (at / 8) + at % 8;
      float gate = 0.f, up = 0.f;
#pragma unroll
      for (int s = 0; s < kLinWaves; ++s) {
        gate += sum[s * kToks * kRows];
        up += sum[s * kToks * kRows + 8];
      }
      if constexpr (kScale) {
        gate *= linear_unscale(base_s[n]);
        up *= linear_unscale(base_s[n]);
      }
      if (a.bias) {
        gate += (float)static_cast<const T*>(a.bias)[f];
        up += (float)static_cast<const T*>(a.bias)[f_all + f];
      }
      static_cast<T*>(a.y)[t * a.ldy + f] = (T)(linear_act(gate, a.act) * up);
    }
    return;
  }
  for (int id = tid; id < kRows * kToks; id += kLinThreads) {
    const int r = row0 + id % kRows, t = tok0 + id / kRows;
    if (r >= a.d_out || t >= a.n_tok) continue;
    float v = 0.f;
#pragma unroll
    for (int s = 0; s < kLinWaves; ++s) v += part[s * kToks * kRows + id];
    if constexpr (kScale) v *= linear_unscale(base_s[id / kRows]);
    if (a.bias) v += (float)static_cast<const T*>(a.bias)[r];
    v = linear_act(v, a.act);
    if (a.residual) v += (float)static_cast<const T*>(a.residual)[t * a.ldr + r];
    static_cast<T*>(a.y)[t * a.ldy + r] = (T)v;
  }
}

__device__ __forceinline__ f32x16_t mfma_32x32x16(u32x4_t a, u32x4_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// One LDS-DMA load: 64 lanes x 16 bytes from `base + voff` (per lane) to the 1 KB of LDS that starts at byte address lds_addr
// (wave-uniform, handed over in M0, which has to be one wait state old when the load reads it: the s_nop).  One outstanding vector-memory
// operation of the wavefront.
__device__ __forceinline__ void lds_dma_1k(const void* base, unsigned voff, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds_addr), "v"(voff), "s"(base) : "memory");
}
// The same with 4 bytes a lane, and with 2, which are zero-extended to 4.
__device__ __forceinline__ void lds_dma_dword(const void* base, unsigned voff, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds_addr), "v"(voff), "s"(base) : "memory");
}
__device__ __forceinline__ void lds_dma_ushort(const void* base, unsigned voff, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %2" : : "s"(lds_addr), "v"(voff), "s"(base) : "memory");
}
// Waits until at most N vector-memory operations are outstanding (the other counters' fields at their maxima).
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt has six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070 | 0x0f00);
}

// Shape of a work-group of the tile kernel: WR x WT wavefronts of RT x TT blocks of 32 rows x 32 tokens, KS times over the columns.
template <int K, int WR_, int WT_, int KS_, int RT_, int TT_, int STAGES_>
struct LinearTile {
  static constexpr int WR = WR_, WT = WT_, KS = KS_, RT = RT_, TT = TT_, kStages = STAGES_;
  static constexpr int kRows = 32 * RT * WR, kToks = 32 * TT * WT;
  static constexpr int kPart = 64 * WR * WT, kThreads = kPart * KS;
  static constexpr int kAcc = 16 * RT * TT;              // accumulators of a lane
  static constexpr int kDma = kToks * 128 / 1024 / (WR * WT);       // requests of a wavefront per 64 columns
  static constexpr int kStage = kToks * 128;             // bytes of 64 columns of X
  static constexpr int kRing = kStages * KS * kStage;
  // a wavefront's own: the coefficients of a group of its rows, and its words, four to a lane, of all its blocks of rows or, where these do not
  // fit, of one block after the other
  static constexpr int kWaves = kThreads / 64;
  static constexpr int kCoefs = (K + 1) * RT * 256;
  static constexpr int kTurns = kRing + kWaves * (kCoefs + K * RT * 1024) <= 160 * 1024 ? 1 : RT;
  static constexpr int kWordBytes = K * RT / kTurns * 1024;
  static constexpr size_t kLds = (size_t)kRing + kWaves * (kCoefs + kWordBytes);
  static_assert(WT == 1, "a row belongs to one wavefront of a part");
  static_assert(kDma % 4 == 0, "a quarter with each step");
  static_assert(kStages >= 3, "the requests of a stage are spread over the one before");
  static_assert(kLds <= 160 * 1024, "one work-group to a CU");
  static_assert(kTurns == 1 || (kTurns == 2 && WR * WT * kWordBytes <= kStage), "the second block's first words wait in the ring's last slot");
  static_assert(KS == 1 || (size_t)(KS / 2) * kRows * kToks * 4 <= kLds, "the joining of the parts has to fit");
};

// X in the order of the tile kernel: images of 32 tokens x 64 columns, [token / 32][chunk of 256 columns][j][4 KB], of words j and 4 + j of the
// chunk (half 0 and 1).  The operand of (token t, half h, step f), 16 bytes, lies at 128 t + 16 ((4 h + f) ^ (t / 2 & 7)): 16 consecutive tokens
// of a step and half fall into all 64 banks of LDS.  Tokens from n_tok on and columns from d_in on are zero (a block's images may go on behind the
// last chunk).
// One wavefront per image.
template <typename T>
__global__ __launch_bounds__(256) void linear_order_kernel(LinearArgs a, int n_image, int images, const uint32_t* __restrict__ base) {
  const int id = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= n_image) return;
  const int block = id / images, at = id % images;       // images: of a block of 32 tokens
  const int half = threadIdx.x & 1, t = (threadIdx.x & 63) >> 1;
  const int word = at / 4 * 8 + 4 * half + at % 4;
  const long tok = 32L * block + t;
  const bool on = tok < a.n_tok && 32 * word < a.d_in;
  const T* x = static_cast<const T*>(a.x) + (on ? tok * a.ldx + 32L * word : 0L);
  uint32_t raw[16];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const u32x4_t v = linear_load8(x + 8 * q, a.vec_x);
#pragma unroll
    for (int e = 0; e < 4; ++e) raw[4 * q + e] = on ? v[e] : 0u;
  }
  if constexpr (!__is_same(T, _Float16)) {
    const uint32_t base2 = on ? base[tok] * 0x10001u : 0u;
#pragma unroll
    for (int e = 0; e < 16; ++e) raw[e] = linear_half2(raw[e], base2);
  }
  u32x4_t step[4];
  plane_order(raw, step);
  u32x4_t* to = static_cast<u32x4_t*>(a.ws) + (long)id * 256 + 8 * t;
#pragma unroll
  for (int f = 0; f < 4; ++f) to[(4 * half + f) ^ (t >> 1 & 7)] = step[f];
}

// Every token's base (linear_base), a wavefront each.
template <typename T>
__global__ __launch_bounds__(256) void linear_base_kernel(LinearArgs a, uint32_t* __restrict__ base) {
  const int tok = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (tok >= a.n_tok) return;
  const T* x = static_cast<const T*>(a.x) + tok * a.ldx;
  uint32_t most = 0;
#pragma unroll 4
  for (int c = 8 * lane; c < a.d_in; c += 512) most = linear_most(linear_load8(x + c, a.vec_x), most);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t b = __shfl_xor(most, o, 64);
    most = most > b ? most : b;
  }
  if (lane == 0) base[tok] = linear_base(most);
}

// Eight rows from `first` of one token: bias, activation, residual, one rounding.
template <typename T, int ACT>
__device__ __forceinline__ void linear_finish8(const LinearArgs& a, long tok, int first, f32x4_t v0, f32x4_t v1,
                                               float unscale, const float (&bias)[8], bool vec_y, bool vec_r) {
  typedef T T8 __attribute__((ext_vector_type(8)));
  float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
  const int n = a.d_out - first < 8 ? a.d_out - first : 8;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = linear_act<ACT>(v[i] * unscale + bias[i]);
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

// Eight values from `first` of one token of the gated product: both biases, activation, product, one rounding.
template <typename T, int ACT>
__device__ __forceinline__ void linear_finish_pairs(const LinearArgs& a, long tok, int first, const f32x4_t (&v)[4], float unscale,
                                                    const float (&bias)[16]) {
  typedef T T8 __attribute__((ext_vector_type(8)));
  const int n = a.d_out / 2 - first < 8 ? a.d_out / 2 - first : 8;
  T8 out;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    out[i] = (T)(linear_act<ACT>(v[i / 4][i % 4] * unscale + bias[i]) * (v[2 + i / 4][i % 4] * unscale + bias[8 + i]));
  T* y = static_cast<T*>(a.y) + tok * a.ldy + first;
  if (a.vec_y && n == 8) {
    *reinterpret_cast<T8*>(y) = out;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) y[i] = out[i];
  }
}

// Y tile of a work-group of wavefronts that share X.  What bounds it: the vector instructions that decode the weights, beside the matrix instructions, which share a SIMD's issue
// (a stage takes about the longer of the two and 0.4 of the shorter), and the last round of tiles.  4096 bf16 tokens, 18944 x 3584 at 2 bits:
// 517 to 612 us from card to card, some 50 of it GELU, 0.91 to 1.08 PFLOP/s (a library product of the dense 16-bit weights takes 500); 333 tokens,
// 8192 x 8192 in groups of 64: 88 us, 0.51 PFLOP/s (192 work-groups of 128 x 128 on 256 CUs, a wavefront to a SIMD, so that neither matrix nor vector
// instructions hide the other's latency).  GATED, 2 x 18944 x 3584: 4096 bf16 tokens at 2 bits 950 to 1000 us, 1.11 to 1.17 PFLOP/s, matrix instructions
// in 62 % of the busy cycles, vector ones in 30 % (ten rounds of work-groups for 9.25 of work); 333 fp16 tokens at 3 bits in groups of 64 132 to 140 us.
//
// GS: words after which a lane's group may change (of the four that it has of a chunk), VEC: the planes go by 16 bytes.
//
// Operands.  X comes in the order of linear_order_kernel, straight from memory into a ring of stages in LDS (LDS-DMA: no registers, no
// instructions but the request); a row's weights for 256 columns are 16 bytes of each plane per lane (half h of a wavefront: words 4 h ..
// of the chunk) and are decoded in registers, a step of 16 columns ahead of its products.  A stage's barrier stands before its last step, when
// every wavefront has read the stage and the next one has landed.
// A row belongs to one wavefront of a part, so its words and coefficients are requested into LDS by the wavefront that needs them, and its lane makes
// the levels of its own rows.  (With the words and coefficients loaded into registers every use waited for all requests behind it, once to a group:
// 333 tokens, 2 x 18944 x 3584 at 3 bits in groups of 64 took 165 us, 148 so; and 355 before tiles that share rows went to one XCD, whose L2 then
// has the lines of their coefficients, of which a group takes two bytes a row: 333 tokens in groups of 128 163 and 123.)
// The compiler does not see the LDS-DMA requests (inline assembly), so the vmcnt waits are written by hand: at most the requests of
// the stages behind the next one may be outstanding.
template <typename T, int K, typename S, int GS, bool VEC, bool GATED>
__global__ __launch_bounds__(S::kThreads) void linear_tiles_kernel(LinearArgs a, int tok_tiles, const uint32_t* __restrict__ base) {
  constexpr int W = kWords, RT = S::RT, TT = S::TT;
  extern __shared__ uint4 lds_raw[];
  char* lds = reinterpret_cast<char*>(lds_raw);
  const int part = __builtin_amdgcn_readfirstlane(threadIdx.x / S::kPart);
  const int tid = threadIdx.x % S::kPart, lane = tid & 63, low = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % S::WR, wt = wave / S::WR;
  // Work-groups are dealt to the eight XCDs in turn, each with an L2 of its own: consecutive tiles, which share rows, go to one XCD.
  int tile = blockIdx.x;
  if (tok_tiles > 1) {
    const int all = gridDim.x / 8, more = gridDim.x % 8, xcd = tile % 8;
    tile = xcd * all + (xcd < more ? xcd : more) + tile / 8;
  }
  const int row0 = tile / tok_tiles * S::kRows, tok0 = tile % tok_tiles * S::kToks;
  const int nw = a.d_in / 32, n_grp = a.d_in / a.group, wpg = a.group / 32;
  const int all_chunks = bpdq_ceil_div(nw, 2 * W);
  const int n_chunk = bpdq_ceil_div(all_chunks, S::KS);  // of a part, the last one maybe past the end

  // a stage: kToks / 32 images; the wavefront requests kDma runs of 1 KB.  Stages past the end take the last image, which is of zeros where a
  // part may come to multiply it: under levels of zero an infinity would become a NaN.
  const int n_image = 4 * all_chunks + (S::KS > 1);
  const char* x_from = static_cast<const char*>(a.ws) + (long)(tok0 / 32) * n_image * 4096;
  unsigned run_from[S::kDma];                            // of a run, in bytes from x_from (all of a tile within 32 bits)
#pragma unroll
  for (int i = 0; i < S::kDma; ++i) {
    const int run = wave * S::kDma + i;
    run_from[i] = (unsigned)(run / 4) * (unsigned)n_image * 4096u + (unsigned)(run % 4) * 1024u;
  }
  // A quarter of a stage's runs: requests in one burst hold the wavefront up.  Stage of this part: chunk stage / 4, word stage % 4.
  auto request = [&](int stage, int ring, int quarter) {
    int at = (stage / W * S::KS + part) * W + stage % W;
    at = at < n_image ? at : n_image - 1;
    const unsigned voff = (unsigned)at * 4096u + 16u * lane;
#pragma unroll
    for (int i = quarter * (S::kDma / 4); i < (quarter + 1) * (S::kDma / 4); ++i)
      lds_dma_1k(x_from, voff + run_from[i], (unsigned)((part * S::kStages + ring) * S::kStage + (wave * S::kDma + i) * 1024));
  };

  const char* w_base[K];
  const char* c_base[K + 1];
  const int base_row = GATED ? 0 : row0;                 // (GATED: a plane is below 4 GB, and offsets are from its first row)
  // the stored row of a tile's row, from base_row
  auto stored = [&](int v) { return GATED ? linear_pair_row(row0 + v, a.d_out / 2) : row0 + v < a.d_out ? v : a.d_out - 1 - row0; };
#pragma unroll
  for (int i = 0; i < K; ++i) w_base[i] = reinterpret_cast<const char*>(a.planes + ((long)i * a.d_out + base_row) * nw);
#pragma unroll
  for (int i = 0; i <= K; ++i) c_base[i] = reinterpret_cast<const char*>(a.coefs + ((long)i * a.d_out + base_row) * n_grp);
  unsigned row[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int at = 32 * (RT * wr + r) + low;
    row[r] = stored(at);
  }
  // Words and coefficients go through LDS too, by the wavefront that needs them, so that every load of the loop is a request whose wait is
  // counted: a load into registers would wait for all requests behind it (the compiler does not count these).
  constexpr int kW = VEC ? W : 1;                        // four words at a time (of a chunk), or one (of a stage)
  constexpr int kTurns = VEC ? S::kTurns : 1, kBlocks = RT / kTurns;       // blocks of rows whose words are in LDS at once
  const unsigned own = (unsigned)(S::kRing + (part * (S::kPart / 64) + wave) * (S::kCoefs + S::kWordBytes));
  const char* own_c = lds + own + 4 * lane;
  auto level_word = [&](int stage) { return 2 * W * (stage / W * S::KS + part) + W * half + stage % W; };
  const unsigned own_w = own + S::kCoefs;
  auto request_w = [&](int stage, int turn, unsigned to) {           // words past the end: the row's first, under levels of zero
    const int word = level_word(stage);
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const unsigned voff = (row[turn * kBlocks + b] * (unsigned)nw + (unsigned)(word < nw ? word : 0)) * 4u;
        if constexpr (VEC) lds_dma_1k(w_base[i], voff, to + (b * K + i) * 1024);
        else lds_dma_dword(w_base[i], voff, to + (b * K + i) * 256);
      }
  };
  auto request_c = [&](int stage) {                      // of the group that begins with the stage's word
    const int word = level_word(stage);
    const unsigned g = (unsigned)(word < nw ? word : 0) / (unsigned)wpg;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i <= K; ++i) lds_dma_ushort(c_base[i], (row[r] * (unsigned)n_grp + g) * 2u, own + (r * (K + 1) + i) * 256);
  };
  uint32_t w_cur[RT][K][kW], w_next[RT][K][kW];
  auto read_w = [&](uint32_t (&w)[RT][K][kW], int turn, unsigned from) {
    const char* p = lds + from + (VEC ? 16 : 4) * lane;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int i = 0; i < K; ++i) {
        if constexpr (VEC) {
          const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p + (b * K + i) * 1024);
#pragma unroll
          for (int j = 0; j < W; ++j) w[turn * kBlocks + b][i][j] = v[j];
        } else {
          w[turn * kBlocks + b][i][0] = *reinterpret_cast<const uint32_t*>(p + (b * K + i) * 256);
        }
      }
  };
  _Float16 c_raw[RT][K + 1];
  auto read_c = [&]() {
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i <= K; ++i) c_raw[r][i] = *reinterpret_cast<const _Float16*>(own_c + (r * (K + 1) + i) * 256);
  };
  PlaneLevels<K> levels[RT], levels_next[RT];
  auto make_levels = [&](PlaneLevels<K> (&to)[RT], int stage) {
    const bool on = level_word(stage) < nw;              // words past the end add nothing
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      PlaneLevels<K> made;
      made.set(c_raw[r]);
#pragma unroll
      for (int n = 0; n < PlaneLevels<K>::kRegs; ++n) {
        to[r].lo[n] = on ? made.lo[n] : 0u;
        to[r].hi[n] = on ? made.hi[n] : 0u;
      }
    }
  };

  f32x16_t acc[RT][TT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[r][t][e] = 0.f;
  u32x4_t b[TT], v[2][RT];
  const char* b_base = lds + part * S::kStages * S::kStage + (32 * TT * wt + low) * 128;
  const int b_slot = (4 * half) ^ (low >> 1 & 7);
  auto read_b = [&](int ring, int f, int t) {
    b[t] = *reinterpret_cast<const u32x4_t*>(b_base + ring * S::kStage + ((b_slot ^ f) * 16) + t * (32 * 128));
  };
  auto decode = [&](int j, int f) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      uint32_t words[K];
#pragma unroll
      for (int i = 0; i < K; ++i) words[i] = w_cur[r][i][VEC ? j : 0];
      v[f & 1][r] = PlaneWord<K>(words).values(levels[r], f);
    }
  };

  const unsigned spare = (unsigned)((part * S::kStages + S::kStages - 1) * S::kStage + wave * S::kWordBytes);      // in the slot requested last
  request_w(0, 0, own_w);
  if (kTurns > 1) request_w(0, 1, spare);
  request_c(0);
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s)
#pragma unroll
    for (int q = 0; q < 4; ++q) request(s, s, q);
  wait_vm<(S::kStages - 1) * S::kDma>();
  asm volatile("" ::: "memory");                         // reads of LDS stay behind the wait
  read_w(w_cur, 0, own_w);
  if (kTurns > 1) read_w(w_cur, 1, spare);
  read_c();
  make_levels(levels, 0);
  wait_vm<(S::kStages - 2) * S::kDma>();
  __syncthreads();                                       // (reads of LDS have their data before it)
  if (!VEC) request_w(1, 0, own_w);
  if (kTurns > 1) request_w(W, 0, own_w);
  request_c(GS);
  request(S::kStages - 1, S::kStages - 1, 0);
#pragma unroll
  for (int t = 0; t < TT; ++t) read_b(0, 0, t);
  decode(0, 0);
  int ring = 0;                                          // stage % kStages
  for (int n = 0; n < n_chunk; ++n) {
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int stage = n * W + j, ring1 = ring + 1 < S::kStages ? ring + 1 : 0;
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        // the next words and coefficients, where they landed a stage ago: beside these products
        const bool turn = (j + 1) % GS == 0;             // the next stage's word begins a group
        if (kTurns > 1 && j == 1 && f == 0) read_w(w_next, 0, own_w);
        if (VEC && j + 1 == W && f == 0) read_w(w_next, kTurns - 1, own_w);
        if (GS > 1 && turn && f == 0) read_c();
        if (GS > 1 && turn && f == 1) make_levels(levels_next, stage + 1);
        if (f == 3) {
          wait_vm<(S::kStages - 2) * S::kDma>();
          asm volatile("" ::: "memory");
          if (!VEC) read_w(w_next, 0, own_w);
          if (!VEC || j + 1 == W) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
              for (int i = 0; i < K; ++i)
#pragma unroll
                for (int e = 0; e < kW; ++e) w_cur[r][i][e] = w_next[r][i][e];
          }
          if (GS == 1) {
            read_c();
            make_levels(levels_next, stage + 1);
          }
          if (turn) {
#pragma unroll
            for (int r = 0; r < RT; ++r) levels[r] = levels_next[r];
          }
          __syncthreads();
          // (before the stage's first requests, so that the next stage's wait is one for these; a chunk's words a stage behind its
          // coefficients, so that the wavefront is held up by fewer requests at once)
          if (!VEC) request_w(stage + 2, 0, own_w);
          else if (kTurns == 1 && j == 0) request_w(stage + W, 0, own_w);
          else if (kTurns > 1 && j == 1) request_w(stage - j + W, 1, own_w);
          else if (kTurns > 1 && j + 1 == W) request_w(stage + 1 + W, 0, own_w);
          if (turn) request_c(stage + 1 + GS);
        }
        // the slot of the stage before is free behind its barrier
        if (f == 3) request(stage + S::kStages, ring, 0);
        else request(stage + S::kStages - 1, ring > 0 ? ring - 1 : S::kStages - 1, f + 1);
        decode(f < 3 ? j : (j + 1) % W, (f + 1) & 3);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
#pragma unroll
          for (int r = 0; r < RT; ++r) acc[r][t] = mfma_32x32x16(v[f & 1][r], b[t], acc[r][t]);
          read_b(f < 3 ? ring : ring1, (f + 1) & 3, t);
        }
#pragma unroll
        for (int t = 0; t < TT; ++t) {                   // RT products, one read, vector instructions beside them
          __builtin_amdgcn_sched_group_barrier(0x8, RT, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x2, 4 * RT, 0);
        }
        __builtin_amdgcn_sched_barrier(0);               // or the loads would sink to where they are needed
      }
      ring = ring1;
    }
  }
  wait_vm<0>();                                          // the last requests have landed before LDS serves the rest
  __syncthreads();

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
  static_assert(RT == 2 && (size_t)S::WR * S::WT * 32 * 64 * 4 <= S::kLds, "16 slots a token");
  f32x4_t* mine = reinterpret_cast<f32x4_t*>(lds) + wave * 32 * 16;
  // (GATED: four lanes a token, a lane eight rows of each projection)
  const int s2 = GATED ? 4 * (lane & 3) : 2 * (lane & 7), first = (row0 + 64 * wr + 4 * s2) / (GATED ? 2 : 1);   // the lane's eight rows
  float bias[GATED ? 16 : 8];
#pragma unroll
  for (int i = 0; i < (GATED ? 16 : 8); ++i) {
    const int at = GATED && i >= 8 ? a.d_out / 2 + first + i - 8 : first + i;
    bias[i] = a.bias && first + i % 8 < (GATED ? a.d_out / 2 : a.d_out) ? (float)static_cast<const T*>(a.bias)[at] : 0.f;
  }
  auto finish = [&](int t, auto act) {
    if constexpr (GATED) {
#pragma unroll 1
      for (int it = 0; it < 2; ++it) {
        const int k = it * 16 + (lane >> 2);
        f32x4_t v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = mine[k * 16 + ((s2 + q) ^ (k & 15))];
        const long tok = tok0 + 32 * (TT * wt + t) + k;
        if (tok < a.n_tok && first < a.d_out / 2)
          linear_finish_pairs<T, act.value>(a, tok, first, v, __is_same(T, _Float16) ? 1.f : linear_unscale(base[tok]), bias);
      }
      return;
    } else {
#pragma unroll 1
    for (int it = 0; it < 4; ++it) {
      const int k = it * 8 + (lane >> 3);
      const f32x4_t v0 = mine[k * 16 + (s2 ^ (k & 15))], v1 = mine[k * 16 + ((s2 + 1) ^ (k & 15))];
      const long tok = tok0 + 32 * (TT * wt + t) + k;
      if (tok < a.n_tok && first < a.d_out)
        linear_finish8<T, act.value>(a, tok, first, v0, v1, __is_same(T, _Float16) ? 1.f : linear_unscale(base[tok]), bias, a.vec_y, a.vec_r);
    }
    }
  };
#pragma unroll 1
  for (int t = 0; t < TT; ++t) {
#pragma unroll
    for (int u = 0; u < TT; ++u) {
      if (u != t) continue;                              // uniform: acc stays in registers
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          mine[low * 16 + ((8 * r + 2 * q + half) ^ (low & 15))] =
              f32x4_t{acc[r][u][4 * q], acc[r][u][4 * q + 1], acc[r][u][4 * q + 2], acc[r][u][4 * q + 3]};
    }
    __builtin_amdgcn_wave_barrier();                     // (LDS serves a wavefront in order)
    switch (a.act) {
      case BPDQ_ACT_RELU: finish(t, std::integral_constant<int, BPDQ_ACT_RELU>()); break;
      case BPDQ_ACT_GELU: finish(t, std::integral_constant<int, BPDQ_ACT_GELU>()); break;
      case BPDQ_ACT_GELU_TANH: finish(t, std::integral_constant<int, BPDQ_ACT_GELU_TANH>()); break;
      case BPDQ_ACT_SILU: finish(t, std::integral_constant<int, BPDQ_ACT_SILU>()); break;
      default: finish(t, std::integral_constant<int, BPDQ_ACT_NONE>()); break;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// rows of the tiles of a call
template <bool GATED>
static int linear_tile_rows(int d_out) { return GATED ? bpdq_ceil_div(d_out / 2, 8) * 16 : d_out; }

template <typename T, int K, typename S, int GS, bool VEC, bool GATED>
static int linear_launch_as(const LinearArgs& a, dim3 grid, int tok_tiles, const uint32_t* base, hipStream_t stream) {
  BPDQ_HIP_TRY((bpdq_lds_limit<&linear_tiles_kernel<T, K, S, GS, VEC, GATED>>(S::kLds)));
  hipLaunchKernelGGL((linear_tiles_kernel<T, K, S, GS, VEC, GATED>), grid, dim3(S::kThreads), S::kLds, stream, a, tok_tiles, base);
  BPDQ_LAUNCH_CHECK();
  return 0;
}

template <typename T, int K, typename S, bool GATED>
static int linear_launch_tiles(const LinearArgs& a, hipStream_t stream) {
  const int images = bpdq_ceil_div(a.d_in, 256) * 4 + (S::KS > 1), blocks = bpdq_ceil_div(a.n_tok, S::kToks) * (S::kToks / 32);
  // behind the images
  uint32_t* base = reinterpret_cast<uint32_t*>(static_cast<char*>(a.ws) + linear_image_bytes(a.n_tok, a.d_in));
  if constexpr (!__is_same(T, _Float16)) {
    hipLaunchKernelGGL((linear_base_kernel<T>), dim3(bpdq_ceil_div(a.n_tok, 4)), dim3(256), 0, stream, a, base);
    BPDQ_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL((linear_order_kernel<T>), dim3(bpdq_ceil_div(images * blocks, 4)), dim3(256), 0, stream, a, images * blocks, images, base);
  BPDQ_LAUNCH_CHECK();
  const int tok_tiles = bpdq_ceil_div(a.n_tok, S::kToks);
  const dim3 grid(bpdq_ceil_div(linear_tile_rows<GATED>(a.d_out), S::kRows) * tok_tiles);
  const int wpg = a.group / 32;
  if (a.vec_w) {
    if (wpg % 4 == 0) return linear_launch_as<T, K, S, 4, true, GATED>(a, grid, tok_tiles, base, stream);
    if (wpg % 2 == 0) return linear_launch_as<T, K, S, 2, true, GATED>(a, grid, tok_tiles, base, stream);
    return linear_launch_as<T, K, S, 1, true, GATED>(a, grid, tok_tiles, base, stream);
  }
  return linear_launch_as<T, K, S, 1, false, GATED>(a, grid, tok_tiles, base, stream);
}

template <typename T, int K, int R, int NT, bool GATED>
static int linear_launch(const LinearArgs& a, hipStream_t stream) {
  const dim3 grid(bpdq_ceil_div(linear_tile_rows<GATED>(a.d_out), 16 * R), bpdq_ceil_div(a.n_tok, 16 * NT));
  hipLaunchKernelGGL((linear_rows_kernel<T, K, R, NT, GATED>), grid, dim3(kLinThreads), 0, stream, a);
  BPDQ_LAUNCH_CHECK();
  return 0;
}

template <typename T, int K, int NT, bool GATED>
static int linear_launch_rows(const LinearArgs& a, int r, hipStream_t stream) {
  if (r == 2) return linear_launch<T, K, 2, NT, GATED>(a, stream);
  if (r == 3) return linear_launch<T, K, 3, NT, GATED>(a, stream);
  if (r == 5) return linear_launch<T, K, 5, NT, GATED>(a, stream);
  if constexpr (NT == 1) {
    if (r == 8) return linear_launch<T, K, 8, NT, GATED>(a, stream);
    return linear_launch<T, K, 1, NT, GATED>(a, stream);
  }
  return BPDQ_ERR_LAUNCH;                                // not offered
}

template <typename T, int K, bool GATED>
static int linear_pick(const LinearArgs& a, hipStream_t stream) {
  const LinearPlan p = linear_plan(a.n_tok, a.d_in, linear_tile_rows<GATED>(a.d_out));
  switch (p.kernel) {
    case kRows1: return linear_launch_rows<T, K, 1, GATED>(a, p.r, stream);
    case kRows2: return linear_launch_rows<T, K, 2, GATED>(a, p.r, stream);
    case kTile256: return linear_launch_tiles<T, K, LinearTile<K, 4, 1, 1, 2, 8, 3>, GATED>(a, stream);
    case kTile256x128: return linear_launch_tiles<T, K, LinearTile<K, 4, 1, 1, 2, 4, 3>, GATED>(a, stream);
    case kTile128: return linear_launch_tiles<T, K, LinearTile<K, 2, 1, 2, 2, 4, 3>, GATED>(a, stream);
    default: return linear_launch_tiles<T, K, LinearTile<K, 2, 1, 4, 2, 2, 3>, GATED>(a, stream);
  }
}

template <int K, bool GATED>
int linear_run(const LinearArgs& a, int dtype, hipStream_t stream) {
  return dtype == BPDQ_F16 ? linear_pick<_Float16, K, GATED>(a, stream) : linear_pick<__bf16, K, GATED>(a, stream);
}

// the gated product for one token and d_in <= kGatedTokenMost (gated_token.hip)
constexpr int kGatedTokenMost = 8192;
int gated_token_run(const LinearArgs& a, int bits, int bf16, hipStream_t stream);

// instantiated in linear_k1.hip to linear_k4.hip, and gated_k1.hip to gated_k4.hip
extern template int linear_run<1, false>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<2, false>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<3, false>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<4, false>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<1, true>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<2, true>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<3, true>(const LinearArgs&, int, hipStream_t);
extern template int linear_run<4, true>(const LinearArgs&, int, hipStream_t);

}  // namespace bpdq
