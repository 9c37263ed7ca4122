// The gated product (linear.h) for one token: the look-ups of gemv.hip, gate and up row of a value by the same wavefront.
//
// What bounds it: the look-ups' vector instructions and LDS reads beside the memory, as there.  2 x 18944 x 3584 at 2 bits in groups of 128, one
// bf16 token: 13.7 us (40 MB, 2.9 TB/s); the few-token kernel of the matrix instructions (linear.h) takes 26, since it decodes weights that one token
// uses once.  Sums are of exact products in fp32, so a weight is not rounded to fp16 here.
#include "gemv.h"
#include "linear.h"

namespace bpdq {

// The 16 partial sums of four consecutive values of x, in table order, to t[0], t[64], ...
__device__ __forceinline__ void gemv_table(float4 v, float* __restrict__ t) {
  const float s01 = v.x + v.y, s23 = v.z + v.w;
  const float e[16] = {0.f,  v.x,       v.y,       s01,       v.z, v.x + v.z, v.y + v.z, s01 + v.z,
                       v.w,  v.x + v.w, v.y + v.w, s01 + v.w, s23, v.x + s23, v.y + s23, s01 + s23};
#pragma unroll
  for (int n = 0; n < 16; ++n) t[n * 64] = e[n];
}

// Sums over the lane's words of each row: C_0 S + sum_i C_i (look-ups), the table at LDS address 0.  (gemv.hip has these loops in its kernel: called
// there, they are scheduled worse, 5000 x 8224 at 4 bits 16 -> 20 us, 18944 x 8320 at 2 bits 23 -> 35.)
template <int K, int W, int NG, int ROWS, bool STRIDED, typename Item>
__device__ __forceinline__ void gemv_rows(const Item& cur, const float* __restrict__ Sw, int n_word, int lane, float (&sum)[ROWS]) {
#pragma unroll
  for (int q = 0; q < ROWS; ++q) sum[q] = 0.f;
  const unsigned base0 = 4u * lane, base1 = 4u * lane + 65536u;
  typedef const __attribute__((address_space(3))) float lds_float;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    if (STRIDED && g > 0 && 64 * g >= n_word) break;       // uniform
    float s = 0.f;
#pragma unroll
    for (int j = g * (W / NG); j < (g + 1) * (W / NG); ++j) s += Sw[j * 64 + lane];
    const bool on = !STRIDED || 64 * g + lane < n_word;
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      float t = fmaf(cur.coef(q, 0, g), s, sum[q]);
#pragma unroll
      for (int i = 0; i < K; ++i) {
        float m = 0.f;                                     // one chain of eight adds per word
#pragma unroll
        for (int j = g * (W / NG); j < (g + 1) * (W / NG); ++j) {
          float mj = 0.f;
          const uint32_t w = cur.w[q][i][j];
          const uint32_t ev = w & 0x0f0f0f0fu, od = (w >> 4) & 0x0f0f0f0fu;
#pragma unroll
          for (int n = 0; n < 8; ++n) {
            // address bytes: 0 = lane, 1 = the nibble, 2 and 3 = upper half of the table or not
            const unsigned off = (unsigned)(n * W + j) * 4096u;
            const unsigned a = __builtin_amdgcn_perm((n & 1) ? od : ev, off >= 65536u ? base1 : base0,
                                                     0x03020000u | (unsigned)((4 + (n >> 1)) << 8));
            mj += *reinterpret_cast<lds_float*>(a + (off & 65535u));
          }
          m += mj;
        }
        t = fmaf(cur.coef(q, i + 1, g), m, t);
      }
      // a word past the end adds nothing, whatever its coefficient (zero times an infinite one is not zero)
      sum[q] = on ? t : sum[q];
    }
  }
  if (!STRIDED && W * lane >= n_word) {
#pragma unroll
    for (int q = 0; q < ROWS; ++q) sum[q] = 0.f;
  }
}

// One chunk: d_in <= 2048 W.  ROWS = 2: an item is both rows; 1: an item is one of them, the gate's first.
template <int K, int W, int NG, int ROWS, bool STRIDED>
__global__ __launch_bounds__(kGemvThreads) void gated_token_kernel(LinearArgs a, int bf16, int passes) {
  extern __shared__ float lds[];
  float* T = lds;                                        // [8][W][16][64], at LDS address 0: the kernel has no other LDS
  float* Sw = lds + 8 * W * 16 * 64;                     // [W][64]: sum of x over each word
  int* size_s = reinterpret_cast<int*>(Sw + W * 64);     // [wavefront]: of its values of x
  constexpr int kSegs = 8 * W, kSegPerThread = (kSegs + kGemvWaves - 1) / kGemvWaves;
  const int nw = a.d_in / 32, n_grp = a.d_in / a.group, wpg = a.group / 32, half = a.d_out / 2;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int step = gridDim.x * kGemvWaves, first = blockIdx.x * kGemvWaves + wave;
  constexpr int kItems = 3 - ROWS;                       // of a pair of rows
  typedef GemvItem<K, W, NG, ROWS, !STRIDED && (NG > 1)> Item;
  Item cur, nxt;
  const GemvPlace<W, STRIDED> at(0, nw, wpg, lane);
  auto fetch = [&](int item, Item& it) {
    int f = first + item / kItems * step;
    f = f < half ? f : half - 1;
    gemv_fetch<K, W, NG, ROWS, STRIDED, true>(a.planes, a.coefs, a.d_out, nw, n_grp, wpg, f + (ROWS == 1 && item % 2 ? half : 0), 0, nw, lane,
                                              at, it);
  };
  // x of the table's segments
  const unsigned short* x = static_cast<const unsigned short*>(a.x);
  unsigned short h[kSegPerThread][4];
#pragma unroll
  for (int s = 0; s < kSegPerThread; ++s) {
    const int id = wave + kGemvWaves * s;                // segment (q, j) = (id / W, id % W)
    const int wl = STRIDED ? 64 * (id % W) + lane : W * lane + id % W;
    const unsigned short* p = x + (id < kSegs && wl < nw ? 32 * wl + 4 * (id / W) : 0);
    if (a.vec_x) *reinterpret_cast<uint2*>(h[s]) = *reinterpret_cast<const uint2*>(p);
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) h[s][e] = p[e];
  }
  fetch(0, cur);                                         // (asked for before x is looked at)
  float4 xv[kSegPerThread];
#pragma unroll
  for (int s = 0; s < kSegPerThread; ++s) {
    const int id = wave + kGemvWaves * s, wl = STRIDED ? 64 * (id % W) + lane : W * lane + id % W;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = bf16 ? __builtin_bit_cast(float, (uint32_t)h[s][e] << 16) : (float)__builtin_bit_cast(_Float16, h[s][e]);
      v[e] = id < kSegs && wl < nw ? v[e] : 0.f;
    }
    xv[s] = make_float4(v[0], v[1], v[2], v[3]);
  }
  // A bf16 token whose largest value is 2^64 or more, or below 2^-24, is taken times a power of two, in tables made anew: its sums would leave fp32,
  // or lose bits among fp32's denormals.  (To look costs 0.2 of 4.4 us at 2 x 3584 x 2048, nothing that shows at 14 us.)
  if (bf16) {
    float most = 0.f;
#pragma unroll
    for (int s = 0; s < kSegPerThread; ++s)
      most = fmaxf(most, fmaxf(fmaxf(fabsf(xv[s].x), fabsf(xv[s].y)), fmaxf(fabsf(xv[s].z), fabsf(xv[s].w))));
    const bool large = __any(most >= 0x1p64f), small = !__any(most >= 0x1p-24f);
    if (lane == 0) size_s[wave] = large ? 2 : small ? 0 : 1;
  }
  float scale = 1.f, unscale = 1.f;
  for (;;) {                                             // once, or twice
#pragma unroll
    for (int s = 0; s < kSegPerThread; ++s) {
      const int id = wave + kGemvWaves * s;
      if (id < kSegs) gemv_table(make_float4(xv[s].x * scale, xv[s].y * scale, xv[s].z * scale, xv[s].w * scale), T + id * 16 * 64 + lane);
    }
    __syncthreads();
    const int size = size_s[lane & (kGemvWaves - 1)];
    if (tid < 64 * W) {
      float sw = 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) sw += T[((q * W + (tid >> 6)) * 16 + 15) * 64 + lane];
      Sw[tid] = sw;
    }
    __syncthreads();
    const bool large = __any(size == 2), small = !__any(size > 0);
    if (!bf16 || scale != 1.f || !(large || small)) break;       // uniform over the work-group
    scale = large ? 0x1p-88f : 0x1p100f;
    unscale = large ? 0x1p88f : 0x1p-100f;
  }
  // the first item is here: or the look-ups below, reached with and without a request ahead of them, would wait for
  // everything in flight (vmcnt 0; the other counters at their maxima)
  __builtin_amdgcn_s_waitcnt(0x0f70);
  float gate = 0.f;
  for (int item = 0; item < passes * kItems; ++item) {
    const int f = first + item / kItems * step;
    if (f >= half) break;                                // uniform over the wavefront
    if (item + 1 < passes * kItems) fetch(item + 1, nxt);
    float v[ROWS];
    gemv_rows<K, W, NG, ROWS, STRIDED>(cur, Sw, nw, lane, v);
#pragma unroll
    for (int q = 0; q < ROWS; ++q)
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) v[q] += __shfl_xor(v[q], o, 64);
    cur = nxt;
    if (ROWS == 1 && item % 2 == 0) {
      gate = v[0];
      continue;
    }
    float up = v[ROWS - 1];
    if (ROWS == 2) gate = v[0];
    gate *= unscale;
    up *= unscale;
    if (lane == 0) {
      if (a.bias) {
        const unsigned short g = static_cast<const unsigned short*>(a.bias)[f], u = static_cast<const unsigned short*>(a.bias)[half + f];
        gate += bf16 ? __builtin_bit_cast(float, (uint32_t)g << 16) : (float)__builtin_bit_cast(_Float16, g);
        up += bf16 ? __builtin_bit_cast(float, (uint32_t)u << 16) : (float)__builtin_bit_cast(_Float16, u);
      }
      const float y = linear_act(gate, a.act) * up;
      if (bf16) static_cast<__bf16*>(a.y)[f] = (__bf16)y;
      else static_cast<_Float16*>(a.y)[f] = (_Float16)y;
    }
  }
}

template <int W>
constexpr size_t gated_lds_bytes() { return gemv_lds_bytes<W>() + kGemvWaves * sizeof(int); }

// Items of both rows where two of them, this one and the next, fit the 128 registers of a 1024-thread work-group.
template <int K, int W, int NG, bool STRIDED>
static int gated_token_launch(const LinearArgs& a, int bf16, hipStream_t stream) {
  constexpr int kRegs = K * W + (K + 1) * (!STRIDED && NG > 1 ? NG / 2 : NG), ROWS = kRegs <= 21 ? 2 : 1;
  BPDQ_HIP_TRY((bpdq_lds_limit<&gated_token_kernel<K, W, NG, ROWS, STRIDED>>(gated_lds_bytes<W>())));
  const int units = bpdq_ceil_div(a.d_out / 2, kGemvWaves), passes = bpdq_ceil_div(units, 256);
  hipLaunchKernelGGL((gated_token_kernel<K, W, NG, ROWS, STRIDED>), dim3(bpdq_ceil_div(units, passes)), dim3(kGemvThreads),
                     gated_lds_bytes<W>(), stream, a, bf16, passes);
  BPDQ_LAUNCH_CHECK();
  return 0;
}

// Words of a lane as in gemv.hip's rule.
template <int K>
static int gated_token_pick(const LinearArgs& a, int bf16, hipStream_t stream) {
  const int nw = a.d_in / 32, wpg = a.group / 32;
  if (nw <= 64) return gated_token_launch<K, 1, 1, false>(a, bf16, stream);
  const int W = nw <= 128 ? 2 : 4, strided = bpdq_ceil_div(nw, 64);
  const bool idle = 8 * strided <= ((K >= 3 || wpg == 1) ? 6 : 5) * W;
  const int per = wpg < W ? W / wpg : 1;                 // groups to a lane
  const bool whole = nw % W == 0 && (wpg % W == 0 || W % wpg == 0) && reinterpret_cast<uintptr_t>(a.planes) % (4 * W) == 0 &&
                     reinterpret_cast<uintptr_t>(a.coefs) % (2 * per) == 0;
  if (W == 2) {
    if (!whole || idle) return gated_token_launch<K, 2, 2, true>(a, bf16, stream);
    return per == 1 ? gated_token_launch<K, 2, 1, false>(a, bf16, stream) : gated_token_launch<K, 2, 2, false>(a, bf16, stream);
  }
  if (!whole || idle) return gated_token_launch<K, 4, 4, true>(a, bf16, stream);
  return per == 1   ? gated_token_launch<K, 4, 1, false>(a, bf16, stream)
         : per == 2 ? gated_token_launch<K, 4, 2, false>(a, bf16, stream)
                    : gated_token_launch<K, 4, 4, false>(a, bf16, stream);
}

int gated_token_run(const LinearArgs& a, int bits, int bf16, hipStream_t stream) {
  switch (bits) {
    case 1: return gated_token_pick<1>(a, bf16, stream);
    case 2: return gated_token_pick<2>(a, bf16, stream);
    case 3: return gated_token_pick<3>(a, bf16, stream);
    default: return gated_token_pick<4>(a, bf16, stream);
  }
}

}  // namespace bpdq
