// The next token of each row of logits, from a given random number u.  With M the row's largest value and T its temperature,
//   w_i = exp((x_i - M) / T);
//   top-k keeps the k largest values, top-p of those, in descending order, the fewest whose weights reach p times theirs in all, min-p what is not
//   below its share of the largest weight (ties: lowest index first);
//   token = the lowest kept index i with  sum of the kept w_j, j <= i  >  u * sum of all kept w_j.
//
// Weights are whole numbers, w 2^43 rounded, from an fp64 exponential, so sums are exact and do not depend on their order: a border is where it is
// however a row is dealt to threads, and a run repeats bit for bit.  The error is 2^-44 of the largest weight for each token.
// Selections are by radix: a histogram of the next bits of an order-preserving key (counts for top-k, weights for top-p, weights by index for
// the draw), then its bin where the running sum reaches the target.
#include "common.h"

namespace bpdq {

constexpr int kSampleThreads = 1024;
constexpr int kSampleVocabMost = 1 << 20;                 // 2^20 weights of at most 2^43 fit into 63 bits
constexpr int kSampleBins = 1024;                         // of indices; keys take 256
constexpr double kSampleOne = 0x1p43;

struct SampleArgs {
  const void* logits;
  const float* u;
  const float* temperature;
  const int* top_k;
  const float* top_p;
  const float* min_p;
  int* token;
  float* prob;
  long ld;
  int n_tok, n_vocab;
};

// Larger values have larger keys; 0: not there (minus infinity, or no number).
__device__ __forceinline__ uint32_t sample_key(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);        // (minus zero is zero)
  const uint32_t k = b >> 31 ? ~b : b | 0x80000000u;
  return x > -__builtin_inff() ? k : 0u;
}
__device__ __forceinline__ float sample_value(uint32_t key) {
  return __builtin_bit_cast(float, key >> 31 ? key & 0x7fffffffu : ~key);
}

// exp((x - M) / T) 2^43, rounded: 2^z by whole powers and the exponential's series for |fraction| <= 1/2 up to degree 11 (6e-15).  per: log2(e) / T.
__device__ __forceinline__ unsigned long long sample_weight(float x, float most, double per) {
  if (x == most) return 1ull << 43;
  const double z = ((double)x - (double)most) * per;
  if (!(z >= -45.0)) return 0;                            // (infinities apart make no number)
  const double n = rint(z), f = (z - n) * 0.69314718055994530942;
  double e = 1.0 / 39916800.0;
  e = fma(e, f, 1.0 / 3628800.0);
  e = fma(e, f, 1.0 / 362880.0);
  e = fma(e, f, 1.0 / 40320.0);
  e = fma(e, f, 1.0 / 5040.0);
  e = fma(e, f, 1.0 / 720.0);
  e = fma(e, f, 1.0 / 120.0);
  e = fma(e, f, 1.0 / 24.0);
  e = fma(e, f, 1.0 / 6.0);
  e = fma(e, f, 0.5);
  e = fma(e, f, 1.0);
  e = fma(e, f, 1.0);
  // the fraction's bits of a double in [2^52, 2^53) are its whole part
  return __builtin_bit_cast(unsigned long long, ldexp(e, 43 + (int)n) + 0x1p52) & ((1ull << 52) - 1);
}

// part * total, up or down to a whole number, exactly; part in [0, 1]
__device__ __forceinline__ unsigned long long sample_share(float part, unsigned long long total, bool up) {
  int e;
  const unsigned long long m = (unsigned long long)(frexpf(part, &e) * 0x1p24f);          // part = m 2^(e - 24)
  const int shift = 24 - e;
  const unsigned __int128 full = (unsigned __int128)m * total;
  if (shift > 100) return up && full > 0;
  const unsigned __int128 whole = full >> shift;
  return (unsigned long long)whole + (up && (whole << shift) != full);
}

typedef unsigned long long u64_t;

struct SampleShared {
  u64_t hist[kSampleBins];
  u64_t part[kSampleThreads / 64];
  u64_t before, value;
  int bin;
};

__device__ __forceinline__ u64_t sample_sum(SampleShared& sh, u64_t v) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((tid & 63) == 0) sh.part[tid >> 6] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < kSampleThreads / 64; ++w) v += sh.part[w];
  return v;
}
__device__ __forceinline__ u64_t sample_max(SampleShared& sh, u64_t v) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const u64_t b = __shfl_xor(v, o, 64);
    v = v > b ? v : b;
  }
  __syncthreads();
  if ((tid & 63) == 0) sh.part[tid >> 6] = v;
  __syncthreads();
  for (int w = 0; w < kSampleThreads / 64; ++w) v = v > sh.part[w] ? v : sh.part[w];
  return v;
}
__device__ __forceinline__ void sample_clear(SampleShared& sh) {
  __syncthreads();
  sh.hist[threadIdx.x] = 0;
  __syncthreads();
}
// The first of `bins` bins, from the top if `down`, where the running sum reaches `target` (>= 1): sh.bin (-1: none), sh.before and sh.value.
__device__ __forceinline__ void sample_find(SampleShared& sh, int bins, bool down, u64_t target) {
  const int tid = threadIdx.x;
  __syncthreads();
  const int bin = down ? bins - 1 - tid : tid;
  const u64_t mine = tid < bins ? sh.hist[bin] : 0;
  u64_t v = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64_t b = __shfl_up(v, o, 64);
    if ((tid & 63) >= o) v += b;
  }
  if ((tid & 63) == 63) sh.part[tid >> 6] = v;
  if (tid == 0) sh.bin = -1;
  __syncthreads();
  for (int w = 0; w < (tid >> 6); ++w) v += sh.part[w];
  if (v >= target && v - mine < target) {
    sh.bin = bin;
    sh.before = v - mine;
    sh.value = mine;
  }
  __syncthreads();
}

// One work-group to a row.
template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  const int tid = threadIdx.x, row = blockIdx.x;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  auto each = [&](auto f) {
    for (int i = tid; i < a.n_vocab; i += kSampleThreads) {
      const uint32_t key = sample_key((float)x[i]);
      if (key) f(key, i);
    }
  };

  u64_t top = 0, live = 0;
  each([&](uint32_t key, int i) {
    const u64_t v = (u64_t)key << 32 | (uint32_t)~i;
    top = top > v ? top : v;
    ++live;
  });
  top = sample_max(sh, top);
  live = sample_sum(sh, live);
  const float temperature = a.temperature ? a.temperature[row] : 1.f;
  if (top == 0 || !(temperature > 0.f)) {                 // uniform: nothing is there, or the largest is asked for
    if (tid == 0) {
      a.token[row] = top ? (int)~(uint32_t)top : -1;
      if (a.prob) a.prob[row] = top ? 1.f : 0.f;
    }
    return;
  }
  const float most = sample_value((uint32_t)(top >> 32));
  const double per = 1.4426950408889634074 / (double)temperature;
  auto weight = [&](uint32_t key) { return sample_weight(sample_value(key), most, per); };

  // kept: keys above tau, and of those at tau the ones up to index last
  uint32_t tau = 1;
  int last = a.n_vocab;
  auto kept = [&](uint32_t key, int i) { return key > tau || (key == tau && i <= last); };
  // of the kept ones with key t, all but the first n go: last becomes the index of the n-th
  auto cut = [&](uint32_t t, u64_t n) {
    int block = 0;
    for (int step = 0; step < 2; ++step) {
      sample_clear(sh);
      each([&](uint32_t key, int i) {
        if (key == t && kept(key, i) && (step == 0 || i / kSampleBins == block))
          atomicAdd(&sh.hist[step == 0 ? i / kSampleBins : i % kSampleBins], 1ull);
      });
      sample_find(sh, kSampleBins, false, n);
      n -= sh.before;
      if (step == 0) block = sh.bin;
    }
    return block * kSampleBins + sh.bin;
  };
  // The key at which the sum of amount(key) over the kept ones, from the largest on, reaches `target`: its value in sh.value, what is above in `above`.
  auto select = [&](u64_t target, u64_t& above, auto amount) {
    uint32_t prefix = 0;
    above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      sample_clear(sh);
      each([&](uint32_t key, int i) {
        if (kept(key, i) && (shift == 24 || key >> (shift + 8) == prefix)) atomicAdd(&sh.hist[key >> shift & 255], amount(key));
      });
      sample_find(sh, 256, true, target - above);
      above += sh.before;
      prefix = prefix << 8 | (uint32_t)sh.bin;
    }
    return prefix;
  };

  const int k = a.top_k ? a.top_k[row] : 0;
  if (k > 0 && (u64_t)k < live) {
    u64_t above;
    const uint32_t t = select((u64_t)k, above, [](uint32_t) { return 1ull; });
    const int at = (u64_t)k - above < sh.value ? cut(t, (u64_t)k - above) : last;
    tau = t;
    last = at;
  }
  const float p = a.top_p ? a.top_p[row] : 1.f;
  if (p < 1.f) {
    u64_t total = 0;
    each([&](uint32_t key, int i) {
      if (kept(key, i)) total += weight(key);
    });
    total = sample_sum(sh, total);
    u64_t target = p > 0.f ? sample_share(p, total, true) : 1, above;
    if (target == 0) target = 1;
    const uint32_t t = select(target, above, weight);
    const u64_t one = weight(t), n = (target - above + one - 1) / one;
    const int at = n * one < sh.value ? cut(t, n) : t == tau ? last : a.n_vocab;
    tau = t;
    last = at;
  }
  const float m = a.min_p ? a.min_p[row] : 0.f;
  const u64_t least = m > 0.f ? (u64_t)ceil(kSampleOne * (double)(m < 1.f ? m : 1.f)) : 1;

  // the draw
  int block = 0;
  u64_t total = 0, target = 0, value = 0;
  for (int step = 0; step < 2; ++step) {
    sample_clear(sh);
    u64_t sum = 0;
    each([&](uint32_t key, int i) {
      if (!kept(key, i) || (step == 1 && i / kSampleBins != block)) return;
      const u64_t w = weight(key);
      if (w < least) return;
      atomicAdd(&sh.hist[step == 0 ? i / kSampleBins : i % kSampleBins], w);
      sum += w;
    });
    if (step == 0) {
      total = sample_sum(sh, sum);
      const float u = a.u[row];
      target = u > 0.f ? sample_share(u < 1.f ? u : 1.f, total, false) + 1 : 1;
      if (target > total) target = total;
    }
    sample_find(sh, kSampleBins, false, target);
    target -= sh.before;
    value = sh.value;
    if (step == 0) block = sh.bin;
  }
  if (tid == 0) {
    a.token[row] = block * kSampleBins + sh.bin;
    if (a.prob) a.prob[row] = (float)((double)value / (double)total);
  }
}

}  // namespace bpdq

using namespace bpdq;

extern "C" size_t bpdq_sample_workspace_bytes(int n_tok, int n_vocab) {
  (void)n_tok;
  (void)n_vocab;
  return 0;
}

extern "C" int bpdq_sample(const void* logits, int n_tok, int n_vocab, long ldl, int dtype, const float* temperature, const int* top_k,
                           const float* top_p, const float* min_p, const float* u, int* token, float* prob, void* ws, size_t ws_bytes,
                           void* stream_) {
  if (n_tok < 0) return -2;
  if (n_vocab <= 0 || n_vocab > kSampleVocabMost) return -3;
  if (dtype != BPDQ_F32 && dtype != BPDQ_F16 && dtype != BPDQ_BF16) return -5;
  if (n_tok == 0) return 0;
  auto odd = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; };
  if (!logits || reinterpret_cast<uintptr_t>(logits) % (dtype == BPDQ_F32 ? 4 : 2)) return -1;
  if (ldl < n_vocab) return -4;
  if (odd(temperature)) return -6;
  if (odd(top_k)) return -7;
  if (odd(top_p)) return -8;
  if (odd(min_p)) return -9;
  if (!u || odd(u)) return -10;
  if (!token || odd(token)) return -11;
  if (odd(prob)) return -12;
  const size_t need = bpdq_sample_workspace_bytes(n_tok, n_vocab);
  if (need && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255))) return -13;
  if (ws_bytes < need) return -14;
  const SampleArgs a = {logits, u, temperature, top_k, top_p, min_p, token, prob, ldl, n_tok, n_vocab};
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (dtype == BPDQ_F32) hipLaunchKernelGGL((sample_row_kernel<float>), dim3(n_tok), dim3(kSampleThreads), 0, stream, a);
  else if (dtype == BPDQ_F16) hipLaunchKernelGGL((sample_row_kernel<_Float16>), dim3(n_tok), dim3(kSampleThreads), 0, stream, a);
  else hipLaunchKernelGGL((sample_row_kernel<__bf16>), dim3(n_tok), dim3(kSampleThreads), 0, stream, a);
  BPDQ_LAUNCH_CHECK();
  return 0;
}
