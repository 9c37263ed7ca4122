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

typedef unsigned long long u64_t;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

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
// Key and index as one number: larger values first, of equal ones the lower index.  A key goes without the bits that all values of the logits' type
// share, so that equal values lie side by side, and bins over a range of places tell their indices apart.
template <typename T>
struct SamplePlace {
  static constexpr int kDrop = __is_same(T, float) ? 0 : __is_same(T, _Float16) ? 13 : 16, kBits = 52 - kDrop;
  static __device__ __forceinline__ u64_t of(uint32_t key, int i) { return (u64_t)(key >> kDrop) << 20 | (u64_t)(kSampleVocabMost - 1 - i); }
  static __device__ __forceinline__ int index(u64_t place) { return kSampleVocabMost - 1 - (int)(place & (kSampleVocabMost - 1)); }
  static __device__ __forceinline__ float value(u64_t place) {
    const uint32_t key = (uint32_t)(place >> 20) << kDrop;
    return sample_value(key >> 31 ? key : key | ((1u << kDrop) - 1));
  }
};

// exp((x - M) / T) 2^43, rounded: 2^z by whole powers and the exponential's series for |fraction| <= 1/2 up to degree 11 (6e-15), without
// branches.  per: log2(e) / T.
__device__ __forceinline__ u64_t sample_weight(float x, float most, double per) {
  // (a difference of infinities is no number, and goes the way of what is too small to count)
  const double z = fmax(((double)x - (double)most) * per, -64.0);
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
  const u64_t w = __builtin_bit_cast(u64_t, ldexp(e, 43 + (int)n) + 0x1p52) & ((1ull << 52) - 1);
  return x == most ? 1ull << 43 : w;
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

// Inclusive sums (MAX: maxima) over the lanes up to each one, by DPP: within rows of 16, then from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64_t sample_dpp(u64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
  return (u64_t)hi << 32 | lo;                            // (lanes without a source: 0)
}
template <bool MAX>
__device__ __forceinline__ u64_t sample_wave_scan(u64_t v) {
  auto join = [](u64_t a, u64_t b) { return MAX ? (a > b ? a : b) : a + b; };
  v = join(v, sample_dpp<0x111, 0xf>(v));                 // row_shr 1, 2, 4, 8
  v = join(v, sample_dpp<0x112, 0xf>(v));
  v = join(v, sample_dpp<0x114, 0xf>(v));
  v = join(v, sample_dpp<0x118, 0xf>(v));
  v = join(v, sample_dpp<0x142, 0xa>(v));                 // row_bcast 15 to rows 1 and 3, 31 to rows 2 and 3
  v = join(v, sample_dpp<0x143, 0xc>(v));
  return v;
}
// the largest of a wavefront's, in its last lane
__device__ __forceinline__ uint32_t sample_wave_most(uint32_t v) {
  auto join = [&](int other) { v = v > (uint32_t)other ? v : (uint32_t)other; };
  join(__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));
  join(__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
  join(__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
  join(__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
  join(__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
  join(__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
  return v;
}
__device__ __forceinline__ u64_t sample_lane(u64_t v, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return (u64_t)hi << 32 | lo;
}

// Sums and maxima over a work-group, and over the threads up to each one: one barrier each, behind which every wavefront scans the
// wavefronts' results by itself.  (These lie in two places in turn: who writes the first again has passed the barrier of the second, which all reach
// behind their reading of the first.)
template <int kThreads>
struct SampleGroup {
  static constexpr int kWaves = kThreads / 64;
  static_assert(kWaves >= 4 && kWaves <= 16, "a row of lanes");
  u64_t (&part)[2][kWaves];
  int turn = 0;
  __device__ __forceinline__ explicit SampleGroup(u64_t (&p)[2][kWaves]) : part(p) {}

  // v: scanned over the wavefront.  Returns the scan over the wavefronts, lane w up to wavefront w.
  template <bool MAX>
  __device__ __forceinline__ u64_t waves(u64_t v) {
    auto join = [](u64_t a, u64_t b) { return MAX ? (a > b ? a : b) : a + b; };
    turn ^= 1;
    if ((threadIdx.x & 63) == 63) part[turn][threadIdx.x >> 6] = v;
    __syncthreads();
    u64_t p = part[turn][threadIdx.x & (kWaves - 1)];
    p = join(p, sample_dpp<0x111, 0xf>(p));
    p = join(p, sample_dpp<0x112, 0xf>(p));
    if (kWaves > 4) p = join(p, sample_dpp<0x114, 0xf>(p));
    if (kWaves > 8) p = join(p, sample_dpp<0x118, 0xf>(p));
    return p;
  }
  __device__ __forceinline__ u64_t sum(u64_t v) { return sample_lane(waves<false>(sample_wave_scan<false>(v)), kWaves - 1); }
  __device__ __forceinline__ u64_t max(u64_t v) { return sample_lane(waves<true>(sample_wave_scan<true>(v)), kWaves - 1); }
  __device__ __forceinline__ u64_t scan(u64_t v, u64_t& total) {
    v = sample_wave_scan<false>(v);
    const u64_t p = waves<false>(v);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    total = sample_lane(p, kWaves - 1);
    return wave > 0 ? v + sample_lane(p, wave - 1) : v;
  }
};

// the running sum at which the token is
__device__ __forceinline__ u64_t sample_draw(float u, u64_t total) {
  const u64_t target = u > 0.f ? sample_share(u < 1.f ? u : 1.f, total, false) + 1 : 1;
  return target < total ? target : total;
}

// A row's values by their place j = index + skew in 16-byte blocks: block j / 8 can be loaded whole, whatever the row's address.
template <typename T>
__device__ __forceinline__ int sample_skew(const T* x) { return (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T) % (16 / sizeof(T))); }

// values at .. at + 7 of a row, minus infinity where it has none
template <typename T>
struct SampleEight {
  alignas(16) T raw[8];
  __device__ __forceinline__ void load(const T* __restrict__ x, int at, int n_vocab) {
    if (at >= 0 && at + 8 <= n_vocab) {
#pragma unroll
      for (int q = 0; q < (int)sizeof(T) / 2; ++q) reinterpret_cast<u32x4_t*>(raw)[q] = reinterpret_cast<const u32x4_t*>(x + at)[q];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) raw[e] = at + e >= 0 && at + e < n_vocab ? x[at + e] : (T)(-__builtin_inff());
    }
  }
  // f(value, index) of what is there, or of all, minus infinity what is not
  template <typename F>
  __device__ __forceinline__ void each(int at, F f) const {
    all(at, [&](float v, int i) {
      if (v > -__builtin_inff()) f(v, i);
    });
  }
  template <typename F>
  __device__ __forceinline__ void all(int at, F f) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) f(fmaxf((float)raw[e] + 0.f, -__builtin_inff()), at + e);     // (minus zero is zero, and what is no number goes)
  }
};

// ---------------------------------------------------------------- rows cut into chunks
//
// A row is cut into chunks, a work-group each, in three launches, and a fourth joins them:
//   top    the chunk's largest value and its index, and the largest values of its turns;
//   hist   how far below the row's largest value its values are: a histogram over 256 steps to an octave (counts where the row asks for top-k,
//          weights where for top-p alone; of the turns' largest values where these bound a small top-k);
//   keep   from the bin where the histogram reaches its target: the sum of the weights above it, and a list of what is in it (of all down to it, where
//          the turns' values bound it, or top-p follows top-k, whose target is known only when the exact top-k is);
//   join   ranks the list, which gives the last one kept; then the chunk, and in it the token, where the running sum reaches u of it.
// All comparisons behind the histogram are on (key, index) as one number, `cut` the least that is kept.  A list that would not fit (kSampleList: flat rows,
// rows of equal values, a very large top_k before top-p) leaves the row to one work-group, which selects by radix over the row itself, some 15 passes:
// right, but 100 to 400 us for 152064 values.
//
// What bounds it: the row's three readings come from the caches but for the first, so it is the chain of four launches (one bf16 row of 152064: 3.0, 4.1,
// 4.8 and 7.2 us, where a large copy would read it in 0.1), and for many rows vector instructions, of which the fp64 exponential is some 25 a value: 64
// fp32 rows of 152064 with mixed requests 47 us (39 MB), 256 fp16 rows of 32003 with top-p and min-p 47 us.  A border found once to a row, by
// its last work-group behind a fence, cost more than every work-group's own search: the fence writes the L2 back (hist 19 -> 126 us).  The search reads sums of
// 12 bins first, 2 KB instead of 24 (256 rows of 32003: keep 16.8 -> 14.7 us, hist 16.0 -> 16.9 for making them).

constexpr int kSampleChunkThreads = 256;
constexpr int kSampleChunkWaves = kSampleChunkThreads / 64;
constexpr int kSampleTurn = kSampleChunkThreads * 8;      // values of a work-group's turn
constexpr int kSampleChunks = 256;                        // of a row, at most
constexpr int kSampleSteps = 12 * 256;                    // 12 octaves of 256, from 2^-5 below the largest value to 2^7
constexpr int kSampleShare = kSampleSteps / kSampleChunkThreads;
static_assert(kSampleShare * kSampleChunkThreads == kSampleSteps, "whole shares");
constexpr int kSampleList = 2048;
constexpr int kSampleRanked = 128;                        // up to here every entry is compared with every other (64 rows with lists of up to 940: 26 us with 512)

static int sample_chunks(int n_vocab, int turns) { return bpdq_ceil_div(n_vocab + 7, turns * kSampleTurn); }        // (with the skew)
static int sample_turns(int n_tok, int n_vocab) {         // of a chunk
  int turns = 1;
  while ((long)n_tok * sample_chunks(n_vocab, turns) > 2048 && turns < 8) ++turns;
  while (sample_chunks(n_vocab, turns) > kSampleChunks) ++turns;
  return turns;
}

// What is known of a row before its exact border.
struct SampleBorder {
  u64_t top;                                              // its largest value
  u64_t target, before;                                   // counts or weights: what is to be reached, and what lies above the bin
  int bin;                                                // of the histogram; kSampleSteps: nothing is bounded
  int all;                                                // the list has everything down to the bin, not only what is in it
};

struct SampleWork {
  u64_t* top;                                             // [row][chunk]
  u64_t* sum;                                             // [row][chunk]
  u64_t* hist;                                            // [row][kSampleSteps]
  u64_t* shares;                                          // [row][kSampleChunkThreads]: sums of the histogram's, kSampleShare bins each
  float* high;                                            // [row][chunk][turn][wavefront] largest values
  u64_t* list;                                            // [row][kSampleList]
  SampleBorder* border;                                   // [row]
  int* count;                                             // [row] of the list; above kSampleList: it did not fit
  int chunks, turns;
};

static size_t sample_work(SampleWork& w, void* ws, int n_tok, int n_vocab) {
  BpdqArena arena(ws);
  w.turns = sample_turns(n_tok, n_vocab);
  w.chunks = sample_chunks(n_vocab, w.turns);
  const size_t n = n_tok;
  w.top = arena.take<u64_t>(n * w.chunks);
  w.sum = arena.take<u64_t>(n * w.chunks);
  w.hist = arena.take<u64_t>(n * kSampleSteps);
  w.shares = arena.take<u64_t>(n * kSampleChunkThreads);
  w.list = arena.take<u64_t>(n * kSampleList);
  w.border = arena.take<SampleBorder>(n);
  w.high = arena.take<float>(n * w.chunks * w.turns * kSampleChunkWaves);
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
template <typename T>
__device__ __forceinline__ SampleAsk sample_ask(const SampleArgs& a, int row, u64_t top) {
  SampleAsk ask;
  const float t = a.temperature ? a.temperature[row] : 1.f;
  ask.draw = top != 0 && t > 0.f;
  ask.most = SamplePlace<T>::value(top);
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

// A chunk's values, the first turn's loaded at once.
template <typename T>
struct SampleChunk {
  const T* x;
  int first, turns, n_vocab;
  SampleEight<T> eight;
  __device__ __forceinline__ SampleChunk(const SampleArgs& a, const SampleWork& w, int row, int chunk)
      : x(static_cast<const T*>(a.logits) + row * a.ld), turns(w.turns), n_vocab(a.n_vocab) {
    first = chunk * turns * kSampleTurn + 8 * (int)threadIdx.x - sample_skew(x);
    eight.load(x, first, n_vocab);
  }
  template <typename F>
  __device__ __forceinline__ void eights(F f) {
    for (int turn = 0; turn < turns; ++turn) {
      const int at = first + turn * kSampleTurn;
      SampleEight<T> next;
      if (turn + 1 < turns) next.load(x, at + kSampleTurn, n_vocab);
      f(eight, at);
      eight = next;
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) {             // f(value, index) of what is there
    eights([&](const SampleEight<T>& v, int at) { v.each(at, f); });
  }
  template <typename F>
  __device__ __forceinline__ void all(F f) {              // of all, minus infinity what is not
    eights([&](const SampleEight<T>& v, int at) { v.all(at, f); });
  }
};

typedef SampleGroup<kSampleChunkThreads> SampleChunkGroup;

// the row's largest, from its chunks'
__device__ __forceinline__ u64_t sample_row_top(const SampleWork& w, int row, SampleChunkGroup& group) {
  return group.max(threadIdx.x < (unsigned)w.chunks ? w.top[(long)row * w.chunks + threadIdx.x] : 0);
}

template <typename T>
__global__ __launch_bounds__(kSampleChunkThreads) void sample_top_kernel(SampleArgs a, SampleWork w, bool bounded) {
  __shared__ u64_t part[2][kSampleChunkWaves];
  SampleChunkGroup group(part);
  const int row = blockIdx.x / w.chunks, chunk = blockIdx.x % w.chunks;
  SampleChunk<T> values(a, w, row, chunk);
  if (bounded) {
    for (int i = chunk * kSampleChunkThreads + threadIdx.x; i < kSampleSteps; i += w.chunks * kSampleChunkThreads)
      w.hist[(long)row * kSampleSteps + i] = 0;
    if (chunk == 0) {
      w.shares[(long)row * kSampleChunkThreads + threadIdx.x] = 0;
      if (threadIdx.x == 0) w.count[row] = 0;
    }
  }
  float most = -__builtin_inff();
  int best_at = 0;
  SampleEight<T> best = values.eight;                     // the eight that have it
  float* high = w.high + (long)blockIdx.x * w.turns * kSampleChunkWaves + (threadIdx.x >> 6);
  values.eights([&](const SampleEight<T>& v, int first) {
    float here = -__builtin_inff();
    v.all(first, [&](float x, int) { here = fmaxf(here, x); });
    if (here > most) {                                    // (indices rise: the first of equal ones stays)
      most = here;
      best = v;
      best_at = first;
    }
    if (bounded) {
      const uint32_t key = sample_wave_most(sample_key(here));
      if ((threadIdx.x & 63) == 63) *high = key ? sample_value(key) : -__builtin_inff();
      high += kSampleChunkWaves;
    }
  });
  int at = 0;
#pragma unroll
  for (int e = 7; e >= 0; --e) at = (float)best.raw[e] == most ? best_at + e : at;
  const u64_t top = group.max(most > -__builtin_inff() ? SamplePlace<T>::of(sample_key(most), at) : 0);
  if (threadIdx.x == 0) w.top[blockIdx.x] = top;
}

// where a histogram reaches its target, by a whole work-group: a thread's share of kSampleShare bins, sum_of(thread) in all; found: two words of LDS
template <typename S, typename F>
__device__ __forceinline__ SampleBorder sample_border(const SampleAsk& ask, u64_t top, SampleChunkGroup& group, u64_t* found, S sum_of, F bin_of) {
  u64_t total;
  const u64_t mine = sum_of((int)threadIdx.x);
  if (threadIdx.x == 0) found[0] = kSampleSteps;
  const u64_t run = group.scan(mine, total);
  SampleBorder s;
  s.top = top;
  s.all = ask.k && ask.p < 1.f;
  s.target = ask.k ? (u64_t)ask.k : sample_share(ask.p, total, true);
  if (s.target == 0) s.target = 1;
  u64_t before = run - mine;
  if (run >= s.target && before < s.target) {
    u64_t hist[kSampleShare];
#pragma unroll
    for (int e = 0; e < kSampleShare; ++e) hist[e] = bin_of(threadIdx.x * kSampleShare + e);
#pragma unroll
    for (int e = 0; e < kSampleShare; ++e) {
      if (before < s.target && before + hist[e] >= s.target) {
        found[0] = threadIdx.x * kSampleShare + e;
        found[1] = before;
      }
      before += hist[e];
    }
  }
  __syncthreads();
  s.bin = (int)found[0];
  s.before = s.bin < kSampleSteps ? found[1] : 0;
  return s;
}

// Where a row asks for few of its largest values, there are as many above the k-th largest of its turns' largest ones: these are counted in place of
// all values, by the row's first work-group, and the list takes what is above.  (If half of the turns hold one of N values, N is 0.69 of
// the turns, 1.4 times their half.)
__device__ __forceinline__ bool sample_few(const SampleWork& w, int k) { return 2L * k <= w.chunks * w.turns * kSampleChunkWaves; }

template <typename T>
__global__ __launch_bounds__(kSampleChunkThreads) void sample_hist_kernel(SampleArgs a, SampleWork w) {
  __shared__ u64_t hist[kSampleSteps];
  __shared__ u64_t part[2][kSampleChunkWaves], found[2];
  SampleChunkGroup group(part);
  const int row = blockIdx.x / w.chunks, chunk = blockIdx.x % w.chunks, highs = w.chunks * w.turns * kSampleChunkWaves;
  const int k = a.top_k && a.top_k[row] > 0 && a.top_k[row] < a.n_vocab ? a.top_k[row] : 0;
  if (k == 0 && !(a.top_p && a.top_p[row] < 1.f)) return;                                      // uniform: nothing to bound
  const bool few = k > 0 && sample_few(w, k);
  if (few && chunk > 0) return;                           // uniform
  SampleChunk<T> values(a, w, row, chunk);
  for (int i = threadIdx.x; i < kSampleSteps; i += kSampleChunkThreads) hist[i] = 0;
  const u64_t top = sample_row_top(w, row, group);        // (its barrier is the histogram's too)
  const SampleAsk ask = sample_ask<T>(a, row, top);
  if (!ask.draw) return;                                  // uniform
  auto share = [&](int thread) {
    u64_t sum = 0;
#pragma unroll
    for (int e = 0; e < kSampleShare; ++e) sum += hist[thread * kSampleShare + e];
    return sum;
  };
  if (few) {
    for (int i = threadIdx.x; i < highs; i += kSampleChunkThreads) {
      const float v = w.high[(long)row * highs + i];
      if (v > -__builtin_inff()) atomicAdd(&hist[sample_step(v, ask.most)], 1ull);
    }
    __syncthreads();
    SampleBorder border = sample_border(ask, top, group, found, share, [&](int i) { return hist[i]; });
    if (border.bin == kSampleSteps) border.bin = kSampleSteps - 1;       // fewer turns than that have values
    border.all = 1;
    if (threadIdx.x == 0) w.border[row] = border;
    return;
  }
  if (ask.k) {                                            // uniform
    values.each([&](float v, int) { atomicAdd(&hist[sample_step(v, ask.most)], 1ull); });
  } else {
    values.eights([&](const SampleEight<T>& v, int at) {
      u64_t add[8];
      int step[8];
      v.all(at, [&](float x, int i) {
        add[i - at] = sample_weight(x, ask.most, ask.per);
        step[i - at] = sample_step(x, ask.most);
      });
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (add[e]) atomicAdd(&hist[step[e]], add[e]);
    });
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kSampleSteps; i += kSampleChunkThreads)
    if (hist[i]) atomicAdd(&w.hist[(long)row * kSampleSteps + i], hist[i]);
  const u64_t sum = share((int)threadIdx.x);
  if (sum) atomicAdd(&w.shares[(long)row * kSampleChunkThreads + threadIdx.x], sum);
}

template <typename T>
__global__ __launch_bounds__(kSampleChunkThreads) void sample_keep_kernel(SampleArgs a, SampleWork w) {
  __shared__ u64_t part[2][kSampleChunkWaves], found[2];
  __shared__ u64_t list[kSampleList];
  __shared__ int count, from;
  SampleChunkGroup group(part);
  const int row = blockIdx.x / w.chunks, chunk = blockIdx.x % w.chunks;
  SampleChunk<T> values(a, w, row, chunk);
  if (threadIdx.x == 0) count = 0;
  const u64_t top = sample_row_top(w, row, group);
  const SampleAsk ask = sample_ask<T>(a, row, top);
  SampleBorder border = {top, 0, 0, kSampleSteps, 0};
  if (ask.k && sample_few(w, ask.k) && ask.draw) {        // uniform
    border = w.border[row];
  } else {
    if (ask.draw && (ask.k || ask.p < 1.f))
      border = sample_border(ask, top, group, found, [&](int thread) { return w.shares[(long)row * kSampleChunkThreads + thread]; },
                             [&](int i) { return w.hist[(long)row * kSampleSteps + i]; });
    if (chunk == 0 && threadIdx.x == 0) w.border[row] = border;
  }
  if (!ask.draw) return;                                  // uniform
  const int bin = border.bin;
  const bool all = border.all;
  u64_t sum = 0;
  auto add = [&](float v) {
    const u64_t one = sample_weight(v, ask.most, ask.per);
    sum += one >= ask.least ? one : 0;
  };
  // what surely weighs less than min-p leaves needs no weight: one of `least` units begins half a unit below, and fp32 is off by less than 2^-10 of an
  // exponent below 2^12, where further down nothing reaches it.  (Halves: the distance of two fp32 values may be twice fp32's largest.)
  const float low = log2f((float)ask.least - 0.5f) - 43.f - 0x1p-8f, per = (float)fmin(2.0 * ask.per, 3.4e38), half = 0.5f * ask.most;
  auto likely = [&](float v) { return !(fmaf(0.5f, v, -half) * per < low); };
  if (bin == kSampleSteps && ask.least == 1) {            // uniform
    values.all([&](float v, int) { add(v); });
  } else if (bin == kSampleSteps) {
    values.all([&](float v, int) {
      if (likely(v)) add(v);
    });
  } else if (ask.k == 0 && ask.least == 1) {              // most may be kept: weights without a branch
    values.eights([&](const SampleEight<T>& v, int at) {
      u64_t one[8];
      int step[8];
      v.all(at, [&](float x, int i) {
        step[i - at] = x > -__builtin_inff() ? sample_step(x, ask.most) : kSampleSteps;
        one[i - at] = sample_weight(x, ask.most, ask.per);
      });
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += step[e] < bin && one[e] >= ask.least ? one[e] : 0;
      v.all(at, [&](float x, int i) {
        if (step[i - at] != bin) return;
        const int to = atomicAdd(&count, 1);
        if (to < kSampleList) list[to] = SamplePlace<T>::of(sample_key(x), i);
      });
    });
  } else {
    values.each([&](float v, int i) {
      const int step = sample_step(v, ask.most);
      if (step > bin) return;
      if (all || step == bin) {
        const int at = atomicAdd(&count, 1);
        if (at < kSampleList) list[at] = SamplePlace<T>::of(sample_key(v), i);
        return;
      }
      if (likely(v)) add(v);
    });
  }
  sum = group.sum(sum);
  if (threadIdx.x == 0) {
    w.sum[blockIdx.x] = sum;
    // (a row's counts add up to 2^20 at most; with a chunk's that did not fit they stay above the list's length)
    from = count ? atomicAdd(&w.count[row], count) : 0;
  }
  if (bin == kSampleSteps) return;                        // uniform: no list
  __syncthreads();
  if (from + count <= kSampleList)
    for (int i = threadIdx.x; i < count; i += kSampleChunkThreads) w.list[(long)row * kSampleList + from + i] = list[i];
}

typedef SampleGroup<kSampleThreads> SampleRowGroup;

struct SampleShared {
  u64_t hist[kSampleBins];
  u64_t part[2][kSampleThreads / 64];
  u64_t place[kSampleRanked], weight[kSampleRanked], above[kSampleRanked];       // of a list
  int rank[kSampleRanked];
  u64_t before, value;
  int bin;
};
static_assert(kSampleBins == kSampleThreads, "a thread to a bin");

// The first bin, from the top if `down`, where the running sum reaches `target` (>= 1): sh.bin (-1: none), sh.before and sh.value.
__device__ __forceinline__ void sample_find(SampleShared& sh, SampleRowGroup& group, bool down, u64_t target) {
  __syncthreads();
  const int bin = down ? kSampleBins - 1 - (int)threadIdx.x : (int)threadIdx.x;
  const u64_t mine = sh.hist[bin];
  u64_t total;
  if (threadIdx.x == 0) sh.bin = -1;
  const u64_t run = group.scan(mine, total);
  if (run >= target && run - mine < target) {
    sh.bin = bin;
    sh.before = run - mine;
    sh.value = mine;
  }
  __syncthreads();
}
__device__ __forceinline__ void sample_clear(SampleShared& sh) {
  __syncthreads();
  sh.hist[threadIdx.x] = 0;
  __syncthreads();
}

// A row by one work-group: every selection by radix, passes over the row itself.
template <typename T>
__device__ __forceinline__ void sample_row(const SampleArgs& a, const SampleAsk& ask, int row, SampleShared& sh, SampleRowGroup& group) {
  const int tid = threadIdx.x;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  const int skew = sample_skew(x);
  auto each = [&](auto f) {                               // f(key, index) of what is there
    for (int at = 8 * tid - skew; at < a.n_vocab; at += 8 * kSampleThreads) {
      SampleEight<T> eight;
      eight.load(x, at, a.n_vocab);
      eight.each(at, [&](float v, int i) { f(sample_key(v), i); });
    }
  };
  auto weight = [&](uint32_t key) { return sample_weight(sample_value(key), ask.most, ask.per); };

  // Kept: places from `cut` on.  The place at which the sum of amount(key) over the kept ones, from the largest on, reaches `target`; 0 if it
  // does not.
  u64_t cut = 0;
  auto select = [&](u64_t target, auto amount) {
    u64_t prefix = 0;
    constexpr int kBits = 10;
    static_assert(kSampleBins == 1 << kBits, "digits");
    for (int shift = (SamplePlace<T>::kBits - 1) / kBits * kBits; shift >= 0; shift -= kBits) {
      sample_clear(sh);
      each([&](uint32_t key, int i) {
        const u64_t place = SamplePlace<T>::of(key, i);
        if (place >= cut && place >> (shift + kBits) == prefix) atomicAdd(&sh.hist[place >> shift & (kSampleBins - 1)], amount(key));
      });
      sample_find(sh, group, true, target);
      if (sh.bin < 0) return (u64_t)0;                    // uniform
      target -= sh.before;
      prefix = prefix << kBits | (u64_t)sh.bin;
    }
    return prefix;
  };

  if (ask.k) cut = select((u64_t)ask.k, [](uint32_t) { return 1ull; });
  if (ask.p < 1.f) {
    u64_t total = 0;
    each([&](uint32_t key, int i) {
      if (SamplePlace<T>::of(key, i) >= cut) total += weight(key);
    });
    const u64_t target = sample_share(ask.p, group.sum(total), true);
    cut = select(target > 0 ? target : 1, weight);
  }
  // the draw: a digit of the index, then the next
  int block = 0;
  u64_t total = 0, target = 0;
  for (int step = 0; step < 2; ++step) {
    sample_clear(sh);
    u64_t sum = 0;
    each([&](uint32_t key, int i) {
      if (SamplePlace<T>::of(key, i) < cut || (step == 1 && i / kSampleBins != block)) return;
      const u64_t w = weight(key);
      if (w < ask.least) return;
      atomicAdd(&sh.hist[step == 0 ? i / kSampleBins : i % kSampleBins], w);
      sum += w;
    });
    if (step == 0) {
      total = group.sum(sum);
      target = sample_draw(a.u[row], total);
    }
    sample_find(sh, group, false, target);
    target -= sh.before;
    if (step == 0) block = sh.bin;
  }
  if (tid == 0) {
    a.token[row] = block * kSampleBins + sh.bin;
    if (a.prob) a.prob[row] = (float)((double)sh.value / (double)total);
  }
}

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_join_kernel(SampleArgs a, SampleWork w) {
  __shared__ SampleShared sh;
  SampleRowGroup group(sh.part);
  constexpr int kEach = kSampleList / kSampleThreads;
  const int tid = threadIdx.x, row = blockIdx.x;
  const SampleBorder border = w.border[row];
  const SampleAsk ask = sample_ask<T>(a, row, border.top);
  if (!ask.draw) {                                        // uniform: nothing is there, or the largest is asked for
    if (tid == 0) {
      a.token[row] = border.top ? SamplePlace<T>::index(border.top) : -1;
      if (a.prob) a.prob[row] = border.top ? 1.f : 0.f;
    }
    return;
  }
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  const int skew = sample_skew(x), span = w.turns * kSampleTurn;
  const int n = border.bin < kSampleSteps ? w.count[row] : 0;
  // (a top-k that keeps everything before a top-p has no histogram of weights)
  if (n > kSampleList || (border.bin == kSampleSteps && ask.k && ask.p < 1.f)) {       // uniform
    sample_row<T>(a, ask, row, sh, group);
    return;
  }
  sh.hist[tid] = tid < w.chunks ? w.sum[(long)row * w.chunks + tid] : 0;
  u64_t cut = 0;
  if (n > 0) {
    // the list, in registers
    u64_t place[kEach], weight[kEach];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      const int i = tid + q * kSampleThreads;
      place[q] = i < n ? w.list[(long)row * kSampleList + i] : 0;
      weight[q] = i < n ? sample_weight(SamplePlace<T>::value(place[q]), ask.most, ask.per) : 0;
    }
    if (n <= kSampleRanked) {
      // everyone's rank and the weight above, the list dealt to the threads of an entry
      const int wide = n <= 64 ? 64 : kSampleRanked, parts = kSampleThreads / wide;
      if (tid < wide) {
        sh.place[tid] = place[0];
        sh.weight[tid] = weight[0];
        sh.above[tid] = 0;
        sh.rank[tid] = 0;
      }
      __syncthreads();
      const int me = tid & (wide - 1), share = bpdq_ceil_div(n, parts), end = (tid / wide + 1) * share;
      const u64_t mine = sh.place[me];
      u64_t above = 0;
      int rank = 0;
#pragma unroll 4
      for (int j = end - share; j < (end < n ? end : n); ++j) {
        const bool larger = sh.place[j] > mine;
        rank += larger;
        above += larger ? sh.weight[j] : 0;
      }
      if (rank) {
        atomicAdd(&sh.rank[me], rank);
        atomicAdd(&sh.above[me], above);
      }
      __syncthreads();
      bool in = tid < n;
      if (in) {
        rank = sh.rank[tid];
        above = sh.above[tid];
      }
      if (border.all) {                                   // the exact top-k, and its top-p
        in = in && rank < ask.k;
        if (ask.p < 1.f) {
          const u64_t target = sample_share(ask.p, group.sum(in ? weight[0] : 0), true);
          in = in && above < (target > 0 ? target : 1);
        }
      } else {
        in = in && border.before + (ask.k ? (u64_t)rank : above) < border.target;
      }
      cut = ~group.max(in ? ~place[0] : 0);
    } else {
      // The place at which the running sum over the list, from the largest on, reaches `target`: 1024 bins over what is left of its range at
      // a time, until a bin holds one.
      u64_t low = 0, high = 0;
#pragma unroll
      for (int q = 0; q < kEach; ++q) {
        if (place[q]) low = low > ~place[q] ? low : ~place[q];
        high = high > place[q] ? high : place[q];
      }
      low = ~group.max(low);
      high = group.max(high);
      const u64_t mine = tid < w.chunks ? sh.hist[tid] : 0;
      auto select = [&](u64_t target, u64_t from, bool count) {
        u64_t lo = low > from ? low : from, hi = high;
        for (;;) {
          const int bits = 64 - __clzll((long long)(hi - lo)), shift = hi == lo || bits <= 10 ? 0 : bits - 10;
          sample_clear(sh);
#pragma unroll
          for (int q = 0; q < kEach; ++q)
            if (place[q] >= lo && place[q] <= hi) atomicAdd(&sh.hist[(place[q] - lo) >> shift], count ? 1ull : weight[q]);
          sample_find(sh, group, true, target);
          if (sh.bin < 0) return lo;                      // there are not so many
          target -= sh.before;
          lo += (u64_t)sh.bin << shift;
          const u64_t end = lo + ((1ull << shift) - 1);
          hi = hi < end ? hi : end;
          int in = 0;
#pragma unroll
          for (int q = 0; q < kEach; ++q) in += place[q] >= lo && place[q] <= hi;
          if (shift == 0 || group.sum(in) <= 1) return lo;
        }
      };
      if (border.all) {
        cut = select((u64_t)ask.k, 0, true);
        if (ask.p < 1.f) {
          u64_t total = 0;
#pragma unroll
          for (int q = 0; q < kEach; ++q)
            if (place[q] >= cut) total += weight[q];
          const u64_t target = sample_share(ask.p, group.sum(total), true);
          cut = select(target > 0 ? target : 1, cut, false);
        }
      } else {
        cut = select(border.target - border.before, 0, ask.k != 0);
      }
      __syncthreads();
      sh.hist[tid] = mine;
      __syncthreads();
    }
#pragma unroll
    for (int q = 0; q < kEach; ++q)
      if (place[q] >= cut && weight[q] >= ask.least)      // (an empty place has no weight)
        atomicAdd(&sh.hist[(SamplePlace<T>::index(place[q]) + skew) / span], weight[q]);
  }
  __syncthreads();
  // the chunk, and in it a thread's consecutive values
  u64_t total, run, mine = sh.hist[tid];
  run = group.scan(mine, total);
  u64_t target = sample_draw(a.u[row], total);
  if (run >= target && run - mine < target) {
    sh.bin = tid;
    sh.before = run - mine;
  }
  __syncthreads();
  target -= sh.before;
  const int each = span / kSampleThreads, first = sh.bin * span + tid * each - skew;
  auto one = [&](int i) -> u64_t {
    if (i < 0 || i >= a.n_vocab) return 0;
    const uint32_t key = sample_key((float)x[i]);
    if (key == 0 || SamplePlace<T>::of(key, i) < cut) return 0;
    const u64_t v = sample_weight(sample_value(key), ask.most, ask.per);
    return v >= ask.least ? v : 0;
  };
  mine = 0;
  for (int e = 0; e < each; ++e) mine += one(first + e);
  u64_t here;
  run = group.scan(mine, here);
  if (run >= target && run - mine < target) {
    run -= mine;
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
  const SampleArgs a = {logits, u, temperature, top_k, top_p, min_p, token, prob, ldl, n_tok, n_vocab};
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (dtype == BPDQ_F32) return sample_launch<float>(a, ws, stream);
  if (dtype == BPDQ_F16) return sample_launch<_Float16>(a, ws, stream);
  return sample_launch<__bf16>(a, ws, stream);
}
