// Y = act(X What^T + bias) + residual from the stored bit-plane format (paper Eq. 1; Sec. 5 discusses serving).
// The weights become operands of the 16-bit matrix instructions in registers (planes.h); they are never written anywhere.
//
// Few tokens: what bounds it is the planes' way from memory (k / 8 bytes per weight) and the vector instructions that turn
// codes into values.  A work-group of eight wavefronts owns 16 R rows and NT tiles of 16 tokens; its wavefronts split the columns, 512 at
// a time: lane (row l % 16, quarter l / 16) loads 16 bytes of each plane, its quarter's 128 columns, and is the operand of that row
// for these columns, whatever the order in which they are contracted.  The partial sums meet in LDS, in the order of the
// wavefronts.
#include "planes.h"

namespace bpdq {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
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
  int vec_x, vec_w;                                      // 16-byte loads of X and of the planes
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
          const u32x4_t v = pw.template values<T>(levels[r], f);
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
  return linear_launch<T, K, 2, 2>(a, stream);
}

template <typename T>
static int linear_by_bits(const LinearArgs& a, int bits, hipStream_t stream) {
  switch (bits) {
    case 1: return linear_pick<T, 1>(a, stream);
    case 2: return linear_pick<T, 2>(a, stream);
    case 3: return linear_pick<T, 3>(a, stream);
    default: return linear_pick<T, 4>(a, stream);
  }
}

}  // namespace bpdq

using namespace bpdq;

extern "C" int bpdq_linear(const uint32_t* planes, const uint16_t* coefs_h, int d_out, int d_in, int bits, int group,
                           const void* X, int n_tok, long ldx, int dtype, const void* bias, int act, const void* residual,
                           long ldr, void* Y, long ldy, void* stream_) {
  if (!planes || (reinterpret_cast<uintptr_t>(planes) & 3)) return -1;
  if (!coefs_h || (reinterpret_cast<uintptr_t>(coefs_h) & 1)) return -2;
  if (d_out <= 0) return -3;
  if (d_in <= 0 || d_in % 32) return -4;
  if (bits < 1 || bits > 4) return -5;
  if (group < 32 || group % 32 || d_in % group) return -6;
  if (n_tok < 0) return -8;
  if (dtype != BPDQ_F16 && dtype != BPDQ_BF16) return -10;
  if (act < BPDQ_ACT_NONE || act > BPDQ_ACT_SILU) return -12;
  if (n_tok == 0) return 0;
  if (!X || (reinterpret_cast<uintptr_t>(X) & 1)) return -7;
  if (ldx < d_in) return -9;
  if (reinterpret_cast<uintptr_t>(bias) & 1) return -11;
  if (reinterpret_cast<uintptr_t>(residual) & 1) return -13;
  if (residual && ldr < d_out) return -14;
  if (!Y || (reinterpret_cast<uintptr_t>(Y) & 1)) return -15;
  if (ldy < d_out) return -16;
  LinearArgs a;
  a.planes = planes;
  a.coefs = reinterpret_cast<const _Float16*>(coefs_h);
  a.x = X;
  a.bias = bias;
  a.residual = residual;
  a.y = Y;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldy = ldy;
  a.d_out = d_out;
  a.d_in = d_in;
  a.group = group;
  a.n_tok = n_tok;
  a.act = act;
  a.vec_x = reinterpret_cast<uintptr_t>(X) % 16 == 0 && ldx % 8 == 0;
  a.vec_w = reinterpret_cast<uintptr_t>(planes) % 16 == 0 && d_in % 128 == 0;
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  return dtype == BPDQ_F16 ? linear_by_bits<_Float16>(a, bits, stream) : linear_by_bits<__bf16>(a, bits, stream);
}
