// What the one-token products from the stored bit-plane format share: what a lane loads of a row (gemv.hip has the method).
#pragma once
#include "common.h"

namespace bpdq {

constexpr int kGemvThreads = 1024;
constexpr int kGemvWaves = kGemvThreads / 64;
constexpr int kGemvRowsSplit = 2 * 8 * 32 * kGemvWaves / 2;   // 4096: up to here one row per wavefront fills the CUs

template <int WPL>
constexpr size_t gemv_lds_bytes() { return (size_t)(8 * WPL * 16 * 64 + WPL * 64) * sizeof(float); }

// Plane words and coefficients of one (chunk, row pass) for this lane, as they come from memory: nothing is
// computed from them before their turn, or the request of the next item would wait for its data.
// W words per lane, NG groups among them.  PACKED: a row's NG halves come as one load.
template <int K, int W, int NG, int ROWS, bool PACKED>
struct GemvItem {
  uint32_t w[ROWS][K][W];
  uint32_t cp[ROWS][K + 1][PACKED ? NG / 2 : 1];
  _Float16 c[ROWS][K + 1][PACKED ? 1 : NG];
  __device__ __forceinline__ float coef(int q, int i, int g) const {
    if constexpr (PACKED) {
      const uint32_t h = cp[q][i][g >> 1];
      return (float)__builtin_bit_cast(_Float16, (unsigned short)((g & 1) ? h >> 16 : h));
    } else {
      return (float)c[q][i][g];
    }
  }
};

// Where a lane's words and their coefficients lie in a row, as byte offsets: one pair per word if STRIDED (word j of
// the lane is word 64 j + lane of the chunk), else one (its words are W lane ...).  The row is the wavefront's, so an
// item's addresses are a scalar and these.  Found once per chunk, but anew for every item if STRIDED: the pairs of four
// words would not fit the registers beside two items.
template <int W, bool STRIDED>
struct GemvPlace {
  static constexpr int kN = STRIDED ? W : 1;
  unsigned word[kN], coef[kN];
  __device__ __forceinline__ GemvPlace(int w0, int n_word, int wpg, int lane) {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int wl = STRIDED ? 64 * j + lane : W * lane;
      // past the end: the chunk's first words (the table is zero there, or the lane's sum is dropped)
      const unsigned wf = w0 + (wl < n_word ? wl : 0);
      word[j] = 4u * wf;
      coef[j] = 2u * (wf / (unsigned)wpg);
    }
  }
};

template <typename T>
__device__ __forceinline__ T gemv_load(const void* base, unsigned byte) {
  return *reinterpret_cast<const T*>(static_cast<const char*>(base) + byte);
}

// Rows r0 ... of the item, or (PAIR) row r0 and the one d_out / 2 behind it.
template <int K, int W, int NG, int ROWS, bool STRIDED, bool PAIR = false>
__device__ __forceinline__ void gemv_fetch(const uint32_t* __restrict__ planes, const _Float16* __restrict__ coefs,
                                           int d_out, int nw, int n_grp, int wpg, int r0, int w0, int n_word, int lane,
                                           const GemvPlace<W, STRIDED>& found,
                                           GemvItem<K, W, NG, ROWS, !STRIDED && (NG > 1)>& it) {
  typedef uint32_t words __attribute__((ext_vector_type(W == 1 ? 2 : W)));
  typedef uint32_t halves __attribute__((ext_vector_type(2)));
  const GemvPlace<W, STRIDED> at = STRIDED ? GemvPlace<W, STRIDED>(w0, n_word, wpg, lane) : found;
#pragma unroll
  for (int j = 0; j < GemvPlace<W, STRIDED>::kN; ++j) {
    if (j > 0 && 64 * j >= n_word) break;          // uniform
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      const long r = PAIR ? r0 + q * (d_out / 2) : r0 + q < d_out ? r0 + q : d_out - 1;
      const uint32_t* p = planes + r * nw;
      const _Float16* c = coefs + r * n_grp;
#pragma unroll
      for (int i = 0; i < K; ++i, p += (long)d_out * nw) {
        if constexpr (STRIDED || W == 1) {
          it.w[q][i][j] = gemv_load<uint32_t>(p, at.word[j]);
        } else {
          const words v = gemv_load<words>(p, at.word[0]);
#pragma unroll
          for (int e = 0; e < W; ++e) it.w[q][i][e] = v[e];
        }
      }
#pragma unroll
      for (int i = 0; i <= K; ++i, c += (long)d_out * n_grp) {
        if constexpr (STRIDED || NG == 1) {
          it.c[q][i][j] = gemv_load<_Float16>(c, at.coef[j]);
        } else if constexpr (NG == 2) {
          it.cp[q][i][0] = gemv_load<uint32_t>(c, at.coef[0]);
        } else {
          const halves v = gemv_load<halves>(c, at.coef[0]);
          it.cp[q][i][0] = v[0];
          it.cp[q][i][1] = v[1];
        }
      }
    }
  }
}

}  // namespace bpdq
