// Root-mean-square norm with the residual's addition:
//   s = x + r,   y = s / sqrt(mean(s^2) + eps) * (offset + w),   and in 8 bits: scale = max(amax |y|, 2^-96) / 127, code = rint(y / scale).
//
// A row stays in registers from its one load to its stores: eight consecutive values to a thread and turn, so that every access is 16 bytes a
// lane and whole lines a wavefront.  Squares are summed in fp64, where neither 3e38 nor 1e-30 leaves the range; from there on fp32, y from the
// unrounded sum.
//
// What bounds it: bytes, and for few rows the launch.  4096 bf16 rows of 8192 with an fp32 residual move 403 MB in 74 us (5.4 TB/s; a large copy
// reaches 4.9 to 5.3 from card to card); 16 x 3584 takes 3.5 us in a graph, 3.9 alone, 100000 x 128 10.  To codes vector instructions bound it, some 24 a value and 72 % of the
// busy cycles, conversions to and from fp64 among them: 1023 x 18944 in groups of 128 19.4 us for 58 MB (3.0 TB/s).
#include "common.h"

namespace bpdq {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kNormMost = 65536;                          // values of a row: 1024 threads of eight turns
constexpr float kNormFloor = 0x1p-96f;                    // the least magnitude a scale is made for, as in the cache

struct NormArgs {
  const void* x;
  const void* residual;
  const void* weight;
  void* sum;
  void* y;
  int8_t* codes;
  float* scales;
  long ldx, ldr, lds, ldy, ldc;
  int n_tok, d, group;
  float offset, eps;
  int vec_x, vec_r, vec_s, vec_w, vec_y;                  // by 16 bytes (codes: by 8)
};

// eight consecutive values as they lie in memory, zeros behind the n-th
template <typename T>
struct NormEight {
  alignas(16) T raw[8];
  __device__ __forceinline__ void load(const T* __restrict__ p, bool vec, int n) {
    if (vec && n >= 8) {
#pragma unroll
      for (int q = 0; q < (int)sizeof(T) / 2; ++q) reinterpret_cast<u32x4_t*>(raw)[q] = reinterpret_cast<const u32x4_t*>(p)[q];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) raw[e] = e < n ? p[e] : (T)0.f;
    }
  }
};
template <typename T>
__device__ __forceinline__ void norm_store8(T* __restrict__ p, bool vec, int n, const float (&v)[8]) {
  if (vec && n >= 8) {
    alignas(16) T raw[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) raw[e] = (T)v[e];
#pragma unroll
    for (int q = 0; q < (int)sizeof(T) / 2; ++q) reinterpret_cast<u32x4_t*>(p)[q] = reinterpret_cast<const u32x4_t*>(raw)[q];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = (T)v[e];
  }
}

// T: X, weight, Y; R: residual and sum; NV: turns of a thread.  blockDim.x = threads of a row, a power of two or whole wavefronts; blockDim.y rows (1
// where a row is more than a wavefront's).
template <typename T, typename R, int NV, bool Q8>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a) {
  const int tid = threadIdx.x, per = blockDim.x, waves = per >> 6;
  const long row = (long)blockIdx.x * blockDim.y + threadIdx.y;
  __shared__ double part_sum[16];
  __shared__ float part_most[16];
  if (row >= a.n_tok) return;                             // whole rows, which no barrier or shuffle crosses
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const R* r = a.residual ? static_cast<const R*>(a.residual) + row * a.ldr : nullptr;
  NormEight<T> w[NV];
  float v[NV][8];
  {
    NormEight<T> in[NV];
    NormEight<R> add[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) in[j].load(x + 8 * (j * per + tid), a.vec_x, a.d - 8 * (j * per + tid));
    if (r) {
#pragma unroll
      for (int j = 0; j < NV; ++j) add[j].load(r + 8 * (j * per + tid), a.vec_r, a.d - 8 * (j * per + tid));
    }
    if (a.weight) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        w[j].load(static_cast<const T*>(a.weight) + 8 * (j * per + tid), a.vec_w, a.d - 8 * (j * per + tid));
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) w[j].raw[e] = (T)1.f;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = r ? (float)in[j].raw[e] + (float)add[j].raw[e] : (float)in[j].raw[e];
  }
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)v[j][e], (double)v[j][e], sum);
  const int lanes = per < 64 ? per : 64;
  for (int o = lanes >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (waves > 1) {
    if ((tid & 63) == 0) part_sum[tid >> 6] = sum;
    __syncthreads();
    sum = 0.0;
    for (int q = 0; q < waves; ++q) sum += part_sum[q];
  }
  double inv_rms = rsqrt(sum / a.d + (double)a.eps);
  if (a.sum) {
    R* s = static_cast<R*>(a.sum) + row * a.lds;
#pragma unroll
    for (int j = 0; j < NV; ++j) norm_store8(s + 8 * (j * per + tid), a.vec_s, a.d - 8 * (j * per + tid), v[j]);
  }
  if (inv_rms < 0x1p-120) {                               // (the same for all of a row) as fp32 it would lose bits
    inv_rms *= 0x1p16;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] *= 0x1p-16f;
  }
  // (the value over the root, at most 256, first: root and weight together may leave fp32 either way)
  const float by = (float)inv_rms;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[j][e] = v[j][e] * by * (a.offset + (float)w[j].raw[e]);
  if constexpr (!Q8) {
    T* y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
    for (int j = 0; j < NV; ++j) norm_store8(y + 8 * (j * per + tid), a.vec_y, a.d - 8 * (j * per + tid), v[j]);
  } else {
    // (values behind the row's end are zero, whatever the weight; a maximum that a NaN goes through, as it may be the weight's alone)
    float most[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      most[j] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) most[j] = __builtin_elementwise_maximum(most[j], fabsf(v[j][e]));
    }
    if (a.group == 0) {
#pragma unroll
      for (int j = 1; j < NV; ++j) most[0] = __builtin_elementwise_maximum(most[0], most[j]);
      for (int o = lanes >> 1; o > 0; o >>= 1) most[0] = __builtin_elementwise_maximum(most[0], __shfl_xor(most[0], o, 64));
      if (waves > 1) {
        if ((tid & 63) == 0) part_most[tid >> 6] = most[0];
        __syncthreads();
        for (int q = 0; q < waves; ++q) most[0] = __builtin_elementwise_maximum(most[0], part_most[q]);
      }
#pragma unroll
      for (int j = 1; j < NV; ++j) most[j] = most[0];
    } else {
      for (int o = a.group / 16; o > 0; o >>= 1) {        // (a group is 4 to 32 lanes, and no more than a row's)
#pragma unroll
        for (int j = 0; j < NV; ++j) most[j] = __builtin_elementwise_maximum(most[j], __shfl_xor(most[j], o, 64));
      }
    }
    const int unit = a.group ? a.group : a.d, n_scale = a.group ? a.d / a.group : 1;
    const bool fine = sum < (double)__builtin_inf();      // no NaN and no infinity in the row
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = 8 * (j * per + tid);
      if (at >= a.d) break;
      const float scale = fine && most[j] < __builtin_inff() ? fmaxf(most[j], kNormFloor) * (1.0f / 127.0f) : __builtin_nanf("");
      if (at % unit == 0) a.scales[row * n_scale + at / unit] = scale;
      const float inv = 1.f / scale;
      // y / scale to the nearest whole number, ties to even, in one rounding: behind 1.5 2^23 it is the low byte (under a scale of NaN: any)
      uint32_t c[8], out[2];
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = __builtin_bit_cast(uint32_t, fmaf(v[j][e], inv, 0x1.8p23f));
#pragma unroll
      for (int q = 0; q < 2; ++q)
        out[q] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[4 * q + 3], c[4 * q + 2], 0x0c0c0400u),
                                       __builtin_amdgcn_perm(c[4 * q + 1], c[4 * q], 0x0c0c0400u), 0x05040100u);
      int8_t* p = a.codes + row * a.ldc + at;
      if (a.vec_y && a.d - at >= 8) {
        *reinterpret_cast<u32x2_t*>(p) = u32x2_t{out[0], out[1]};
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at + e < a.d) p[e] = (int8_t)c[e];
      }
    }
  }
}

template <typename T, typename R, int NV, bool Q8>
static int norm_launch(const NormArgs& a, hipStream_t stream) {
  const int turns = bpdq_ceil_div(bpdq_ceil_div(a.d, 8), NV);
  int per = 64;
  if (turns > 64) per = bpdq_ceil_div(turns, 64) * 64;
  else
    while (per > 4 && per / 2 >= turns && 4 * per >= a.group) per /= 2;      // (a group's lanes are a row's)
  const int rows = per > 64 ? 1 : 256 / per;
  if (((long)a.n_tok + rows - 1) / rows * (per * rows) > 0xffffffffL) return -2;       // threads along the grid's x
  hipLaunchKernelGGL((norm_kernel<T, R, NV, Q8>), dim3((unsigned)(((long)a.n_tok + rows - 1) / rows)), dim3(per, rows), 0, stream, a);
  BPDQ_LAUNCH_CHECK();
  return 0;
}

// Turns of a thread, measured (us; bf16, with a residual in bf16, back to back in a graph): few rows want threads, 16 x 3584 3.5 with one
// turn, 3.8 with two, but 333 x 8192 6.4 and 5.5; many rows two, 4096 x 8192 + fp32 79 with one, 75 with two and with four; wide rows so many that a
// CU holds more than two of them: 1023 x 18944 25 to codes and 32 to 16 bits with four turns (640 threads), 19 and 27 with five (512), 21 and 28 with six,
// 35 and 39 with eight; 655 x 29568 24.7 and 32.7, 24.1 and 31.9 (768 threads), 25.4 and 32.4, 29.8 and 34.8.  (Not everywhere: 787 x 24576 to codes takes 28 with
// five, 21 with six.)
template <typename T, typename R, bool Q8>
static int norm_pick(const NormArgs& a, hipStream_t stream) {
  const int vecs = bpdq_ceil_div(a.d, 8);
  if (vecs <= 512 && a.n_tok <= 512) return norm_launch<T, R, 1, Q8>(a, stream);
  if (vecs <= 2048) return norm_launch<T, R, 2, Q8>(a, stream);
  if (vecs <= 5120) return norm_launch<T, R, 5, Q8>(a, stream);
  return norm_launch<T, R, 8, Q8>(a, stream);
}

template <bool Q8>
static int norm_by_type(const NormArgs& a, int dtype, int rdtype, hipStream_t stream) {
  if (dtype == BPDQ_F32) return norm_pick<float, float, Q8>(a, stream);
  if (dtype == BPDQ_F16)
    return rdtype == BPDQ_F16 ? norm_pick<_Float16, _Float16, Q8>(a, stream) : norm_pick<_Float16, float, Q8>(a, stream);
  return rdtype == BPDQ_BF16 ? norm_pick<__bf16, __bf16, Q8>(a, stream) : norm_pick<__bf16, float, Q8>(a, stream);
}

static bool norm_vec(const void* p, long ld, size_t size, size_t unit = 16) {
  return reinterpret_cast<uintptr_t>(p) % unit == 0 && (size_t)ld * size % unit == 0;
}
static bool norm_type(int dtype) { return dtype == BPDQ_F32 || dtype == BPDQ_F16 || dtype == BPDQ_BF16; }

// what both entries check and fill in; a negative code, or 0, or 1 where there is nothing to do
static int norm_args(NormArgs& a, const void* X, int n_tok, int d, long ldx, int dtype, const void* residual, long ldr, int rdtype,
                     void* S, long lds, const void* weight, float offset, float eps) {
  if (n_tok < 0) return -2;
  if (d <= 0 || d > kNormMost) return -3;
  if (!norm_type(dtype)) return -5;
  if (residual && rdtype != dtype && rdtype != BPDQ_F32) return -8;
  if (!(offset - offset == 0.f)) return -12;
  if (!(eps >= 0x1p-126f) || !(eps - eps == 0.f)) return -13;
  if (n_tok == 0) return 1;
  const size_t size = dtype == BPDQ_F32 ? 4 : 2, wide = residual && rdtype == BPDQ_F32 ? 4 : size;
  if (!X || reinterpret_cast<uintptr_t>(X) % size) return -1;
  if (ldx < d) return -4;
  if (reinterpret_cast<uintptr_t>(residual) % wide) return -6;
  if (residual && ldr < d) return -7;
  if (S && (!residual || reinterpret_cast<uintptr_t>(S) % wide)) return -9;
  if (S && lds < d) return -10;
  if (reinterpret_cast<uintptr_t>(weight) % size) return -11;
  a = NormArgs{};
  a.x = X;
  a.residual = residual;
  a.weight = weight;
  a.sum = S;
  a.ldx = ldx;
  a.ldr = ldr;
  a.lds = lds;
  a.n_tok = n_tok;
  a.d = d;
  a.offset = offset;
  a.eps = eps;
  a.vec_x = norm_vec(X, ldx, size);
  a.vec_r = norm_vec(residual, ldr, wide);
  a.vec_s = norm_vec(S, lds, wide);
  a.vec_w = norm_vec(weight, 0, size);
  return 0;
}

}  // namespace bpdq

using namespace bpdq;

extern "C" int bpdq_rms_norm(const void* X, int n_tok, int d, long ldx, int dtype, const void* residual, long ldr, int rdtype,
                             void* S, long lds, const void* weight, float offset, float eps, void* Y, long ldy, void* stream) {
  NormArgs a;
  const int rc = norm_args(a, X, n_tok, d, ldx, dtype, residual, ldr, rdtype, S, lds, weight, offset, eps);
  if (rc) return rc < 0 ? rc : 0;
  const size_t size = dtype == BPDQ_F32 ? 4 : 2;
  if (!Y || reinterpret_cast<uintptr_t>(Y) % size) return -14;
  if (ldy < d) return -15;
  a.y = Y;
  a.ldy = ldy;
  a.vec_y = norm_vec(Y, ldy, size);
  return norm_by_type<false>(a, dtype, residual ? rdtype : dtype, static_cast<hipStream_t>(stream));
}

extern "C" int bpdq_rms_norm_q8(const void* X, int n_tok, int d, long ldx, int dtype, const void* residual, long ldr, int rdtype,
                                void* S, long lds, const void* weight, float offset, float eps, int group, int8_t* codes, long ldc,
                                float* scales, void* stream) {
  NormArgs a;
  const int rc = norm_args(a, X, n_tok, d, ldx, dtype, residual, ldr, rdtype, S, lds, weight, offset, eps);
  if (rc < 0) return rc;
  if (group != 0 && ((group != 32 && group != 64 && group != 128 && group != 256) || d % group)) return -14;
  if (rc) return 0;
  if (!codes) return -15;
  if (ldc < d) return -16;
  if (!scales || (reinterpret_cast<uintptr_t>(scales) & 3)) return -17;
  a.codes = codes;
  a.scales = scales;
  a.ldc = ldc;
  a.group = group;
  a.vec_y = norm_vec(codes, ldc, 1, 8);
  return norm_by_type<true>(a, dtype, residual ? rdtype : dtype, static_cast<hipStream_t>(stream));
}
