// Weights as fp16 operands of the matrix instructions, straight from the stored bit-plane format (paper Eq. 1).
//
// A group's 2^k levels of a row, ((C_0 + b_1 C_1) + b_2 C_2) + ... in fp32 in this order, rounded once to fp16 (11 bits; the coefficients
// are halves themselves, so small sums are exact), lie in registers as two tables of bytes (low and high halves), and v_perm_b32, which picks four bytes out of eight by four
// selector bytes, turns four codes into four low or high bytes at once.
//
// The codes of four columns as bytes come from the plane words by a shift and a mask if the columns are eight apart, so the 32
// columns of a word are taken in the order
//   step f = 0..3:  2f, 2f + 8, 2f + 16, 2f + 24, 2f + 1, 2f + 9, 2f + 17, 2f + 25
// (the contraction does not care), and the other operand is brought into the same order by plane_order().
// Per weight 0.6 to 2 vector instructions for the codes (two planes: their even bits and their odd bits are merged first, whole
// words at a time) and one for the tables.
#pragma once
#include "common.h"

namespace bpdq {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t bit_select(uint32_t mask, uint32_t a, uint32_t b) { return (a & mask) | (b & ~mask); }

// The levels of one (row, group).
template <int K>
struct PlaneLevels {
  static constexpr int kRegs = K <= 2 ? 1 : 1 << (K - 2);
  uint32_t lo[kRegs], hi[kRegs];

  __device__ __forceinline__ void set(const _Float16 (&c)[K + 1]) {
    uint32_t v[1 << K];
#pragma unroll
    for (int n = 0; n < (1 << K); ++n) {
      float s = (float)c[0];
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (n >> i & 1) s += (float)c[i + 1];
      v[n] = __builtin_bit_cast(unsigned short, (_Float16)s);
    }
#pragma unroll
    for (int r = 0; r < kRegs; ++r) {
      uint32_t a, b;                                     // levels 4r, 4r + 1 and 4r + 2, 4r + 3 side by side
      a = v[4 * r] | v[4 * r + 1] << 16;
      b = K == 1 ? a : v[(4 * r + 2) & ((1 << K) - 1)] | v[(4 * r + 3) & ((1 << K) - 1)] << 16;
      lo[r] = __builtin_amdgcn_perm(b, a, 0x06040200u);
      hi[r] = __builtin_amdgcn_perm(b, a, 0x07050301u);
    }
  }

  // four codes (bytes) to four values, in two words
  __device__ __forceinline__ void take(uint32_t code, uint32_t& first, uint32_t& second) const {
    uint32_t l, h;
    if constexpr (K <= 2) {
      l = __builtin_amdgcn_perm(lo[0], lo[0], code);
      h = __builtin_amdgcn_perm(hi[0], hi[0], code);
    } else if constexpr (K == 3) {
      l = __builtin_amdgcn_perm(lo[1], lo[0], code);
      h = __builtin_amdgcn_perm(hi[1], hi[0], code);
    } else {
      const uint32_t upper = ((code >> 3) & 0x01010101u) * 0xffu, low3 = code & 0x07070707u;
      l = bit_select(upper, __builtin_amdgcn_perm(lo[3], lo[2], low3), __builtin_amdgcn_perm(lo[1], lo[0], low3));
      h = bit_select(upper, __builtin_amdgcn_perm(hi[3], hi[2], low3), __builtin_amdgcn_perm(hi[1], hi[0], low3));
    }
    first = __builtin_amdgcn_perm(h, l, 0x05010400u);
    second = __builtin_amdgcn_perm(h, l, 0x07030602u);
  }
};

// The plane words of 32 columns, their bits merged two planes at a time.
template <int K>
struct PlaneWord {
  uint32_t even[(K + 1) / 2], odd[(K + 1) / 2];          // codes of the even and of the odd columns, two bits each (one plane: as it is)
  __device__ __forceinline__ explicit PlaneWord(const uint32_t (&w)[K]) {
#pragma unroll
    for (int p = 0; p < K; p += 2) {
      if (p + 1 < K) {
        even[p / 2] = bit_select(0x55555555u, w[p], w[p + 1] << 1);
        odd[p / 2] = bit_select(0x55555555u, w[p] >> 1, w[p + 1]);
      } else {
        even[p / 2] = w[p];
        odd[p / 2] = w[p] >> 1;
      }
    }
  }
  __device__ __forceinline__ uint32_t codes(const uint32_t (&v)[(K + 1) / 2], int f) const {
    const uint32_t first = (v[0] >> (2 * f)) & (K == 1 ? 0x01010101u : 0x03030303u);
    if constexpr (K <= 2) return first;
    else return first | ((v[1] >> (2 * f)) & (K == 3 ? 0x01010101u : 0x03030303u)) << 2;
  }
  // the eight values of step f
  __device__ __forceinline__ u32x4_t values(const PlaneLevels<K>& levels, int f) const {
    uint32_t a, b, c, d;
    levels.take(codes(even, f), a, b);
    levels.take(codes(odd, f), c, d);
    return u32x4_t{a, b, c, d};
  }
};

// 32 consecutive 16-bit values (x[q]: values 2q, 2q + 1) to the four steps' operands
__device__ __forceinline__ void plane_order(const uint32_t (&x)[16], u32x4_t (&step)[4]) {
#pragma unroll
  for (int f = 0; f < 4; ++f)
    step[f] = u32x4_t{__builtin_amdgcn_perm(x[f + 4], x[f], 0x05040100u), __builtin_amdgcn_perm(x[f + 12], x[f + 8], 0x05040100u),
                      __builtin_amdgcn_perm(x[f + 4], x[f], 0x07060302u), __builtin_amdgcn_perm(x[f + 12], x[f + 8], 0x07060302u)};
}

}  // namespace bpdq
