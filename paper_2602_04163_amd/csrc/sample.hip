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
constexpr int kSampleRowsMost = 1 << 15;                  // times 256 chunks of 256 threads: within the grid's 2^32
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
  int n_tok, n_vocab, vec;
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
  u64_t part[kSampleThreads / 64 + 2];
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

// ---------------------------------------------------------------- rows cut into chunks
//
// A row is cut into chunks, a work-group each, in three launches, and a fourth joins them:
//   top    the chunk's largest value and its index;
//   hist   how far below the row's largest value its values are: a histogram over 256 steps to an octave (counts where the row asks for top-k,
//          weights where for top-p alone);
//   keep   from the bin where the histogram reaches its target: the sum of the weights above it, and a list of what is in it (of all down to it, where
//          top-p follows top-k, because its target is known only when the exact top-k is);
//   join   ranks the list, which gives the last one kept; then the chunk, and in it the token, where the running sum reaches u of it.
// All comparisons behind the histogram are on (key, index) as one number, `cut` the least that is kept.  A list that would not fit (kSampleList: flat rows,
// rows of equal values, a very large top_k before top-p) leaves the row to one work-group, which selects by radix over the row itself.

constexpr int kSampleChunkThreads = 256;
constexpr int kSampleTurn = kSampleChunkThreads * 8;      // values of a work-group's turn
constexpr int kSampleChunks = 256;                        // of a row, at most
constexpr int kSampleSteps = 3072;                        // 12 octaves of 256, from 2^-5 below the largest value to 2^7
constexpr int kSampleList = 2048;

__host__ __device__ static inline int sample_turns(int n_tok, int n_vocab) {       // of a chunk
  int turns = 1;
  while ((long)n_tok * bpdq_ceil_div(n_vocab, turns * kSampleTurn) > 2048 && turns < 8) ++turns;
  while (bpdq_ceil_div(n_vocab, turns * kSampleTurn) > kSampleChunks) ++turns;
  return turns;
}

struct SampleWork {
  u64_t* top;                                             // [row][chunk]
  u64_t* sum;                                             // [row][chunk]
  u64_t* hist;                                            // [row][kSampleSteps]
  u64_t* list;                                            // [row][kSampleList]
  int* count;                                             // [row] of the list; above kSampleList: it did not fit
  int chunks, turns;
};

static size_t sample_work(SampleWork& w, void* ws, int n_tok, int n_vocab) {
  BpdqArena arena(ws);
  w.turns = sample_turns(n_tok, n_vocab);
  w.chunks = bpdq_ceil_div(n_vocab, w.turns * kSampleTurn);
  const size_t n = n_tok;
  w.top = arena.take<u64_t>(n * w.chunks);
  w.sum = arena.take<u64_t>(n * w.chunks);
  w.hist = arena.take<u64_t>(n * kSampleSteps);
  w.list = arena.take<u64_t>(n * kSampleList);
  w.count = arena.take<int>(n);
  return arena.off;
}

// How a row's values are bounded.
struct SampleAsk {
  float most;                                             // the row's largest value
  double per;                                             // log2(e) / T
  int k;                                                  // 0: no top-k
  float p;                                                // 1: no top-p
  u64_t least;                                            // the least weight that min-p leaves
  bool draw;                                              // not: the largest value is the answer
};
__device__ __forceinline__ SampleAsk sample_ask(const SampleArgs& a, int row, u64_t top) {
  SampleAsk ask;
  const float t = a.temperature ? a.temperature[row] : 1.f;
  ask.draw = top != 0 && t > 0.f;
  ask.most = sample_value((uint32_t)(top >> 32));
  ask.per = 1.4426950408889634074 / (double)t;
  const int k = a.top_k ? a.top_k[row] : 0;
  ask.k = k > 0 && k < a.n_vocab ? k : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  ask.p = p < 1.f ? (p > 0.f ? p : 0.f) : 1.f;
  const float m = a.min_p ? a.min_p[row] : 0.f;
  ask.least = m > 0.f ? (u64_t)ceil(kSampleOne * (double)(m < 1.f ? m : 1.f)) : 1;
  return ask;
}

// the bin of a value so far below the largest
__device__ __forceinline__ int sample_step(float x, float most) {
  if (x == most) return 0;                                // (infinities too)
  const int step = (int)(__builtin_bit_cast(uint32_t, most - x) >> 15) - ((127 - 5) << 8);
  return step < 0 ? 0 : step < kSampleSteps ? step : kSampleSteps - 1;
}

// f(value, index) of the chunk's values that are there
template <typename T, typename F>
__device__ __forceinline__ void sample_each(const SampleArgs& a, const T* __restrict__ x, int first, int end, bool vec, F f) {
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  for (int at = first + 8 * threadIdx.x; at < end; at += 8 * blockDim.x) {
    alignas(16) T raw[8];
    if (vec && at + 8 <= end) {
#pragma unroll
      for (int q = 0; q < (int)sizeof(T) / 2; ++q) reinterpret_cast<u32x4_t*>(raw)[q] = reinterpret_cast<const u32x4_t*>(x + at)[q];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) raw[e] = at + e < end ? x[at + e] : (T)(-__builtin_inff());
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = (float)raw[e] + 0.f;                // (minus zero is zero)
      if (v > -__builtin_inff()) f(v, at + e);
    }
  }
}

template <typename V, typename F>
__device__ __forceinline__ V sample_fold(V v, V* part, F f) {        // over a work-group of kSampleChunkThreads
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = f(v, (V)__shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < kSampleChunkThreads / 64; ++w) v = f(v, part[w]);
  return v;
}
__device__ __forceinline__ u64_t sample_larger(u64_t a, u64_t b) { return a > b ? a : b; }
__device__ __forceinline__ u64_t sample_add(u64_t a, u64_t b) { return a + b; }

// the row's largest, from its chunks'
__device__ __forceinline__ u64_t sample_row_top(const SampleWork& w, int row, u64_t* part) {
  const u64_t mine = threadIdx.x < (unsigned)w.chunks ? w.top[(long)row * w.chunks + threadIdx.x] : 0;
  return sample_fold(mine, part, sample_larger);
}

template <typename T>
__global__ __launch_bounds__(kSampleChunkThreads) void sample_top_kernel(SampleArgs a, SampleWork w, bool clear) {
  __shared__ u64_t part[kSampleChunkThreads / 64];
  const int row = blockIdx.x / w.chunks, chunk = blockIdx.x % w.chunks, first = chunk * w.turns * kSampleTurn;
  const int end = first + w.turns * kSampleTurn < a.n_vocab ? first + w.turns * kSampleTurn : a.n_vocab;
  u64_t top = 0;
  sample_each(a, static_cast<const T*>(a.logits) + row * a.ld, first, end, a.vec, [&](float v, int i) {
    top = sample_larger(top, (u64_t)sample_key(v) << 32 | (uint32_t)~i);
  });
  top = sample_fold(top, part, sample_larger);
  if (threadIdx.x == 0) w.top[blockIdx.x] = top;
  if (clear) {
    for (int i = chunk * kSampleChunkThreads + threadIdx.x; i < kSampleSteps; i += w.chunks * kSampleChunkThreads)
      w.hist[(long)row * kSampleSteps + i] = 0;
    if (chunk == 0 && threadIdx.x == 0) w.count[row] = 0;
  }
}

template <typename T>
__global__ __launch_bounds__(kSampleChunkThreads) void sample_hist_kernel(SampleArgs a, SampleWork w) {
  __shared__ u64_t hist[kSampleSteps];
  __shared__ u64_t part[kSampleChunkThreads / 64];
  const int row = blockIdx.x / w.chunks, chunk = blockIdx.x % w.chunks, first = chunk * w.turns * kSampleTurn;
  const int end = first + w.turns * kSampleTurn < a.n_vocab ? first + w.turns * kSampleTurn : a.n_vocab;
  const SampleAsk ask = sample_ask(a, row, sample_row_top(w, row, part));
  if (!ask.draw || (ask.k == 0 && ask.p == 1.f)) return; // uniform
  for (int i = threadIdx.x; i < kSampleSteps; i += kSampleChunkThreads) hist[i] = 0;
  __syncthreads();
  sample_each(a, static_cast<const T*>(a.logits) + row * a.ld, first, end, a.vec, [&](float v, int) {
    const u64_t add = ask.k ? 1 : sample_weight(v, ask.most, ask.per);
    if (add) atomicAdd(&hist[sample_step(v, ask.most)], add);
  });
  __syncthreads();
  for (int i = threadIdx.x; i < kSampleSteps; i += kSampleChunkThreads)
    if (hist[i]) atomicAdd(&w.hist[(long)row * kSampleSteps + i], hist[i]);
}

// What the histogram says of a row.
struct SampleBorder {
  u64_t target, before;                                   // counts or weights: what is to be reached, and what lies above the bin
  int bin;                                                // kSampleSteps: everything is kept
};
// by a whole work-group of `threads`; part: threads / 64 + 3 words of LDS
__device__ __forceinline__ SampleBorder sample_border(const SampleWork& w, const SampleAsk& ask, int row, u64_t* part, int threads) {
  const int each = bpdq_ceil_div(kSampleSteps, threads), waves = threads / 64, tid = threadIdx.x;
  const u64_t* hist = w.hist + (long)row * kSampleSteps;
  u64_t mine = 0;
  for (int e = 0; e < each; ++e)
    if (tid * each + e < kSampleSteps) mine += hist[tid * each + e];
  u64_t run = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64_t b = __shfl_up(run, o, 64);
    if ((tid & 63) >= o) run += b;
  }
  __syncthreads();
  if ((tid & 63) == 63) part[tid >> 6] = run;
  if (tid == 0) part[waves] = kSampleSteps;
  __syncthreads();
  u64_t total = 0;
  for (int q = 0; q < waves; ++q) {
    if (q == tid >> 6) run += total;
    total += part[q];
  }
  SampleBorder s;
  s.target = ask.k ? (u64_t)ask.k : sample_share(ask.p, total, true);
  if (s.target == 0) s.target = 1;
  if (run >= s.target && run - mine < s.target) {
    u64_t before = run - mine;
    for (int e = 0; e < each; ++e) {
      const u64_t here = hist[tid * each + e];
      if (before + here >= s.target) {
        part[waves] = tid * each + e;
        part[waves + 1] = before;
        break;
      }
      before += here;
    }
  }
  __syncthreads();
  s.bin = (int)part[waves];
  s.before = s.bin < kSampleSteps ? part[waves + 1] : 0;
  return s;
}

template <typename T>
__global__ __launch_bounds__(kSampleChunkThreads) void sample_keep_kernel(SampleArgs a, SampleWork w) {
  __shared__ u64_t part[kSampleChunkThreads / 64 + 2];
  __shared__ u64_t list[kSampleList];
  __shared__ int count, from;
  const int row = blockIdx.x / w.chunks, chunk = blockIdx.x % w.chunks, first = chunk * w.turns * kSampleTurn;
  const int end = first + w.turns * kSampleTurn < a.n_vocab ? first + w.turns * kSampleTurn : a.n_vocab;
  const SampleAsk ask = sample_ask(a, row, sample_row_top(w, row, part));
  if (!ask.draw) return;                                  // uniform
  int bin = kSampleSteps;
  if (ask.k || ask.p < 1.f) bin = sample_border(w, ask, row, part, kSampleChunkThreads).bin;
  const bool all = ask.k && ask.p < 1.f;                  // the whole top-k goes to the list
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  u64_t sum = 0;
  sample_each(a, static_cast<const T*>(a.logits) + row * a.ld, first, end, a.vec, [&](float v, int i) {
    const int step = bin < kSampleSteps ? sample_step(v, ask.most) : 0;
    if (step > bin) return;
    if (bin < kSampleSteps && (all || step == bin)) {
      const int at = atomicAdd(&count, 1);
      if (at < kSampleList) list[at] = (u64_t)sample_key(v) << 32 | (uint32_t)~i;
      return;
    }
    const u64_t one = sample_weight(v, ask.most, ask.per);
    if (one >= ask.least) sum += one;
  });
  sum = sample_fold(sum, part, sample_add);
  if (threadIdx.x == 0) {
    w.sum[blockIdx.x] = sum;
    // (a chunk's count is at most 2^20 and a row's 2^20, so the sum with a chunk that did not fit stays above the list's length)
    from = count ? atomicAdd(&w.count[row], count) : 0;
  }
  __syncthreads();
  if (from + count <= kSampleList)
    for (int i = threadIdx.x; i < count; i += kSampleChunkThreads) w.list[(long)row * kSampleList + from + i] = list[i];
}

// the running sum at which the token is
__device__ __forceinline__ u64_t sample_draw(float u, u64_t total) {
  const u64_t target = u > 0.f ? sample_share(u < 1.f ? u : 1.f, total, false) + 1 : 1;
  return target < total ? target : total;
}

// A row by one work-group: every selection by radix, passes over the row itself.
template <typename T>
__device__ __noinline__ void sample_row(const SampleArgs& a, const SampleAsk& ask, int row, SampleShared& sh) {
  const int tid = threadIdx.x;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  auto each = [&](auto f) {
    for (int i = tid; i < a.n_vocab; i += kSampleThreads) {
      const uint32_t key = sample_key((float)x[i]);
      if (key) f(key, i);
    }
  };

  u64_t live = 0;
  each([&](uint32_t, int) { ++live; });
  live = sample_sum(sh, live);
  auto weight = [&](uint32_t key) { return sample_weight(sample_value(key), ask.most, ask.per); };

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

  const int k = ask.k;
  if (k > 0 && (u64_t)k < live) {
    u64_t above;
    const uint32_t t = select((u64_t)k, above, [](uint32_t) { return 1ull; });
    const int at = (u64_t)k - above < sh.value ? cut(t, (u64_t)k - above) : last;
    tau = t;
    last = at;
  }
  if (ask.p < 1.f) {
    u64_t total = 0;
    each([&](uint32_t key, int i) {
      if (kept(key, i)) total += weight(key);
    });
    total = sample_sum(sh, total);
    u64_t target = sample_share(ask.p, total, true), above;
    if (target == 0) target = 1;
    const uint32_t t = select(target, above, weight);
    const u64_t one = weight(t), n = (target - above + one - 1) / one;
    const int at = n * one < sh.value ? cut(t, n) : t == tau ? last : a.n_vocab;
    tau = t;
    last = at;
  }
  // the draw
  int block = 0;
  u64_t total = 0, target = 0, value = 0;
  for (int step = 0; step < 2; ++step) {
    sample_clear(sh);
    u64_t sum = 0;
    each([&](uint32_t key, int i) {
      if (!kept(key, i) || (step == 1 && i / kSampleBins != block)) return;
      const u64_t w = weight(key);
      if (w < ask.least) return;
      atomicAdd(&sh.hist[step == 0 ? i / kSampleBins : i % kSampleBins], w);
      sum += w;
    });
    if (step == 0) {
      total = sample_sum(sh, sum);
      target = sample_draw(a.u[row], total);
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


template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_join_kernel(SampleArgs a, SampleWork w) {
  __shared__ SampleShared sh;
  __shared__ u64_t list[kSampleList], weights[kSampleList];
  static_assert(kSampleChunks <= kSampleBins && kSampleThreads >= kSampleChunks, "a row's chunks are a histogram's bins");
  const int tid = threadIdx.x, row = blockIdx.x;
  const u64_t top = sample_max(sh, tid < w.chunks ? w.top[(long)row * w.chunks + tid] : 0);
  const SampleAsk ask = sample_ask(a, row, top);
  if (!ask.draw) {                                        // uniform: nothing is there, or the largest is asked for
    if (tid == 0) {
      a.token[row] = top ? (int)~(uint32_t)top : -1;
      if (a.prob) a.prob[row] = top ? 1.f : 0.f;
    }
    return;
  }
  u64_t cut = 0;
  sh.hist[tid] = tid < w.chunks ? w.sum[(long)row * w.chunks + tid] : 0;
  if (ask.k || ask.p < 1.f) {
    const SampleBorder border = sample_border(w, ask, row, sh.part, kSampleThreads);
    const int n = border.bin < kSampleSteps ? w.count[row] : 0;
    // a top-k that keeps everything before a top-p has no histogram of weights
    if (n > kSampleList || (border.bin == kSampleSteps && ask.k && ask.p < 1.f)) {
      sample_row<T>(a, ask, row, sh);
      return;
    }
    for (int i = tid; i < n; i += kSampleThreads) {
      list[i] = w.list[(long)row * kSampleList + i];
      weights[i] = sample_weight(sample_value((uint32_t)(list[i] >> 32)), ask.most, ask.per);
    }
    __syncthreads();
    // ranks in the list, and the weight above
    constexpr int kEach = kSampleList / kSampleThreads;
    int rank[kEach];
    u64_t above[kEach];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      rank[q] = 0;
      above[q] = 0;
      const int i = tid + q * kSampleThreads;
      if (i >= n) continue;
      const u64_t mine = list[i];
      for (int j = 0; j < n; ++j)
        if (list[j] > mine) {
          ++rank[q];
          above[q] += weights[j];
        }
    }
    u64_t target = border.target, before = border.before;
    const bool all = ask.k && ask.p < 1.f;
    if (all) {                                            // of the exact top-k
      u64_t total = 0;
#pragma unroll
      for (int q = 0; q < kEach; ++q)
        if (tid + q * kSampleThreads < n && rank[q] < ask.k) total += weights[tid + q * kSampleThreads];
      total = sample_sum(sh, total);
      target = sample_share(ask.p, total, true);
      if (target == 0) target = 1;
      before = 0;
    }
    u64_t last = ~0ull;
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      const int i = tid + q * kSampleThreads;
      if (i >= n) continue;
      const bool in = all ? rank[q] < ask.k && above[q] < target : ask.k ? before + rank[q] < target : before + above[q] < target;
      if (!in) continue;
      last = last < list[i] ? last : list[i];
      if (weights[i] >= ask.least) atomicAdd(&sh.hist[(int)~(uint32_t)list[i] / (w.turns * kSampleTurn)], weights[i]);
    }
    cut = ~sample_max(sh, ~last);                         // the smallest of the kept ones
    if (border.bin == kSampleSteps) cut = 0;
  }
  __syncthreads();
  u64_t total = sample_sum(sh, sh.hist[tid]);
  u64_t target = sample_draw(a.u[row], total);
  sample_find(sh, w.chunks, false, target);
  target -= sh.before;
  // in the chunk: a thread's consecutive values
  const int span = w.turns * kSampleTurn, each = span / kSampleThreads, first = sh.bin * span + tid * each;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  auto one = [&](int i) -> u64_t {
    if (i >= a.n_vocab) return 0;
    const uint32_t key = sample_key((float)x[i]);
    if (key == 0 || ((u64_t)key << 32 | (uint32_t)~i) < cut) return 0;
    const u64_t v = sample_weight(sample_value(key), ask.most, ask.per);
    return v >= ask.least ? v : 0;
  };
  u64_t mine = 0;
  for (int e = 0; e < each; ++e) mine += one(first + e);
  __syncthreads();
  sh.hist[tid] = mine;
  sample_find(sh, kSampleThreads, false, target);
  if (tid == sh.bin) {
    u64_t run = sh.before;
    for (int e = 0; e < each; ++e) {
      const u64_t v = one(first + e);
      run += v;
      if (run >= target) {
        a.token[row] = first + e;
        if (a.prob) a.prob[row] = (float)((double)v / (double)total);
        break;
      }
    }
  }
}

template <typename T>
static int sample_launch(const SampleArgs& a, void* ws, hipStream_t stream) {
  SampleWork w;
  sample_work(w, ws, a.n_tok, a.n_vocab);
  const bool bounded = a.top_k || a.top_p;
  const dim3 grid((unsigned)a.n_tok * w.chunks), block(kSampleChunkThreads);
  hipLaunchKernelGGL((sample_top_kernel<T>), grid, block, 0, stream, a, w, bounded);
  BPDQ_LAUNCH_CHECK();
  if (bounded) {
    hipLaunchKernelGGL((sample_hist_kernel<T>), grid, block, 0, stream, a, w);
    BPDQ_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL((sample_keep_kernel<T>), grid, block, 0, stream, a, w);
  BPDQ_LAUNCH_CHECK();
  hipLaunchKernelGGL((sample_join_kernel<T>), dim3(a.n_tok), dim3(kSampleThreads), 0, stream, a, w);
  BPDQ_LAUNCH_CHECK();
  return 0;
}

}  // namespace bpdq

using namespace bpdq;

extern "C" size_t bpdq_sample_workspace_bytes(int n_tok, int n_vocab) {
  if (n_tok <= 0 || n_tok > kSampleRowsMost || n_vocab <= 0 || n_vocab > kSampleVocabMost) return 0;
  SampleWork w;
  return sample_work(w, nullptr, n_tok, n_vocab);
}

extern "C" int bpdq_sample(const void* logits, int n_tok, int n_vocab, long ldl, int dtype, const float* temperature, const int* top_k,
                           const float* top_p, const float* min_p, const float* u, int* token, float* prob, void* ws, size_t ws_bytes,
                           void* stream_) {
  if (n_tok < 0 || n_tok > kSampleRowsMost) return -2;
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
  const int vec = reinterpret_cast<uintptr_t>(logits) % 16 == 0 && (size_t)ldl * (dtype == BPDQ_F32 ? 4 : 2) % 16 == 0;
  const SampleArgs a = {logits, u, temperature, top_k, top_p, min_p, token, prob, ldl, n_tok, n_vocab, vec};
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (dtype == BPDQ_F32) return sample_launch<float>(a, ws, stream);
  if (dtype == BPDQ_F16) return sample_launch<_Float16>(a, ws, stream);
  return sample_launch<__bf16>(a, ws, stream);
}
