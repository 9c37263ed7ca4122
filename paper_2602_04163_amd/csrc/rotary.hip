// Rotary positions: channel pair i of a head at position p is turned by the angle p f_i,
//   (a, b) -> m (a cos - b sin, b cos + a sin),    pairs (i, i + rot / 2) or (2 i, 2 i + 1), i < rot / 2; channels from rot on pass.
//
// Angles are formed in fp64 as turns, p f / 2 pi, of which only the fraction counts: at position 10^6 an fp32 angle would be off by 0.06.  The
// fraction, as fp32 good to 2^-26 of a turn, goes to sincospif.  A work-group makes the angles of its tokens once, in LDS, for all heads of Q and K.
//
// What bounds it: bytes, and for few tokens the launch.  8192 fp16 tokens of 72 heads of 128 move 302 MB in 50 us (5.9 TB/s on buffers that the caches
// hold in part, 64 us with new ones); 37 ragged chunks of 20 heads of 64, half of each turned, 74 MB in 14 us (5.2 TB/s); 16 tokens of 32 heads take 3.2 us in a graph.
// Requests of several heads at once (two, four) cost more in registers than they gain: 51 us became 52 and 60.
#include "common.h"

namespace bpdq {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kRotThreads = 256;
constexpr int kRotPer = 4;                                // tokens of a work-group at most
constexpr int kRotDimMost = 512;

struct RotaryArgs {
  const double* freq;
  const int* pos;
  const int* tok_start;
  const void* q;
  const void* k;
  void* q_out;
  void* k_out;
  long ldq, ldk, ldqo, ldko;
  int rot, half, n_tok, max_tok, n_q, n_kv, dim, per;     // half: pairs (i, i + rot / 2)
  int copy_q, copy_k;                                     // channels from rot on have to be written (not where the call is in place)
  float mscale, sign;
};

// E consecutive channels at once
template <typename T, int E>
struct RotaryUnit {
  alignas(E * sizeof(T)) T v[E];
};

// a c + b s, with the same roundings whichever units a call takes: left to itself the compiler fuses the last one into the conversion to fp16 in
// some of them.
__device__ __forceinline__ float rotary_turn(float a, float c, float b, float s) {
  float sum = fmaf(a, c, b * s);
  asm("" : "+v"(sum));
  return sum;
}

// E: channels of a unit (of pairs that lie apart: of both their halves); 1: single pairs and channels.
template <typename T, int E>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 turn[kRotPer * kRotDimMost / 2];
  typedef RotaryUnit<T, E> Unit;
  const int tid = threadIdx.x, seq = blockIdx.y, pairs = a.rot / 2;
  const long p0 = a.pos[seq], first = a.tok_start[seq];
  long n = (long)a.tok_start[seq + 1] - first;
  n = n < a.max_tok ? n : a.max_tok;
  n = n < a.n_tok - first ? n : a.n_tok - first;
  const long from = (long)blockIdx.x * a.per;
  if (p0 < 0 || first < 0 || from >= n) return;           // uniform
  const int toks = n - from < a.per ? (int)(n - from) : a.per;

  for (int id = tid; id < toks * pairs; id += kRotThreads) {
    const int t = id / pairs, i = id - t * pairs;
    const double turns = (double)(p0 + from + t) * a.freq[i] * 0.15915494309189533577;
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    turn[id] = float2{a.mscale * c, a.sign * a.mscale * s};
  }
  __syncthreads();

  // units of a head: those of pairs, then those that pass; its (token, head)s come to the threads of a unit in turn
  const bool apart = a.half || E == 1;                    // a unit has the first channels of its pairs, and the second ones elsewhere
  const int paired = apart ? pairs / E : a.rot / E, units = paired + (a.dim - a.rot) / E;
  const int wide = units < kRotThreads ? units : kRotThreads;
  const int slot = tid / wide, slots = kRotThreads / wide, heads = a.n_q + a.n_kv;
  if (slot >= slots) return;
  const int step_t = slots / heads, step_h = slots - step_t * heads;
  const int near = a.half ? pairs : 1;                    // from the first channel of a pair to the second
  for (int u = tid % wide; u < units; u += wide) {
    const bool turned = u < paired;
    const int ch = !turned ? a.rot + (u - paired) * E : E == 1 && !a.half ? 2 * u : u * E;      // the unit's first channel
    int h = slot % heads;
    for (int t = slot / heads; t < toks;) {
      const bool is_q = h < a.n_q;
      if (turned || (is_q ? a.copy_q : a.copy_k)) {
        const long row = first + from + t;
        const T* p = (is_q ? static_cast<const T*>(a.q) + row * a.ldq + h * a.dim
                           : static_cast<const T*>(a.k) + row * a.ldk + (h - a.n_q) * a.dim) + ch;
        T* to = (is_q ? static_cast<T*>(a.q_out) + row * a.ldqo + h * a.dim
                      : static_cast<T*>(a.k_out) + row * a.ldko + (h - a.n_q) * a.dim) + ch;
        Unit x = *reinterpret_cast<const Unit*>(p);
        if (turned && apart) {
          Unit y = *reinterpret_cast<const Unit*>(p + near);
          const float2* angle = turn + t * pairs + u * E;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float c = angle[e].x, s = angle[e].y, one = (float)x.v[e], two = (float)y.v[e];
            x.v[e] = (T)(rotary_turn(one, c, -two, s));
            y.v[e] = (T)(rotary_turn(two, c, one, s));
          }
          *reinterpret_cast<Unit*>(to + near) = y;
        } else if (turned) {
          const float2* angle = turn + t * pairs + u * (E / 2);
#pragma unroll
          for (int e = 0; e + 1 < E; e += 2) {
            const float c = angle[e / 2].x, s = angle[e / 2].y, one = (float)x.v[e], two = (float)x.v[e + 1];
            x.v[e] = (T)(rotary_turn(one, c, -two, s));
            x.v[e + 1] = (T)(rotary_turn(two, c, one, s));
          }
        }
        *reinterpret_cast<Unit*>(to) = x;
      }
      h += step_h;
      t += step_t;
      if (h >= heads) {
        h -= heads;
        ++t;
      }
    }
  }
}

template <typename T, int E>
static int rotary_as(const RotaryArgs& a, int n_seq, hipStream_t stream) {
  hipLaunchKernelGGL((rotary_kernel<T, E>), dim3(bpdq_ceil_div(a.max_tok, a.per), n_seq), dim3(kRotThreads), 0, stream, a);
  BPDQ_LAUNCH_CHECK();
  return 0;
}

// Units of 16 bytes where pairs, heads, rows and addresses are whole ones, of two channels where they are whole twos, else single ones: 4000 bf16
// tokens of 40 heads of 80, 20 of these turned: 30 us by single ones.
template <typename T>
static int rotary_launch(const RotaryArgs& a, int n_seq, hipStream_t stream) {
  auto whole = [&](int e) {
    auto rows = [&](const void* p, long ld, int heads) {
      return heads == 0 || (reinterpret_cast<uintptr_t>(p) % (e * sizeof(T)) == 0 && ld % e == 0);
    };
    return a.dim % e == 0 && (a.half ? a.rot / 2 : a.rot) % e == 0 && rows(a.q, a.ldq, a.n_q) && rows(a.k, a.ldk, a.n_kv) &&
           rows(a.q_out, a.ldqo, a.n_q) && rows(a.k_out, a.ldko, a.n_kv);
  };
  constexpr int kWhole = 16 / (int)sizeof(T);
  if (whole(kWhole)) return rotary_as<T, kWhole>(a, n_seq, stream);
  if (whole(2)) return rotary_as<T, 2>(a, n_seq, stream);
  return rotary_as<T, 1>(a, n_seq, stream);
}

}  // namespace bpdq

using namespace bpdq;

extern "C" int bpdq_rotary_frequencies(int rot, double base, int scaling, double factor, double low, double high, int original,
                                       double* freq, double* mscale) {
  if (rot <= 0 || rot % 2) return -1;
  if (!(base > 1.0) || !(base < 1e300)) return -2;
  if (scaling < BPDQ_ROTARY_PLAIN || scaling > BPDQ_ROTARY_BANDS) return -3;
  if (scaling != BPDQ_ROTARY_PLAIN && (!(factor >= 1.0) || !(factor < 1e300))) return -4;
  const bool by_turns = scaling == BPDQ_ROTARY_YARN || scaling == BPDQ_ROTARY_BANDS;
  if (by_turns && !(low > 0.0)) return -5;
  if (by_turns && (!(high > low) || !(high < 1e300))) return -6;
  if (by_turns && original <= 0) return -7;
  if (!freq) return -8;
  if (scaling == BPDQ_ROTARY_NTK && rot == 2) return -1;  // its one frequency does not depend on the base
  const double two_pi = 6.283185307179586476925;
  if (scaling == BPDQ_ROTARY_NTK) base *= pow(factor, (double)rot / (rot - 2));
  // pair at which a channel makes so many turns in `original` positions
  auto pair_of = [&](double turns) { return rot * log(original / (two_pi * turns)) / (2.0 * log(base)); };
  double ramp_lo = 0.0, ramp_hi = 1.0;
  if (scaling == BPDQ_ROTARY_YARN) {
    ramp_lo = fmax(floor(pair_of(high)), 0.0);
    ramp_hi = fmin(ceil(pair_of(low)), rot - 1.0);
    if (!(ramp_hi > ramp_lo)) ramp_hi = ramp_lo + 0.001;
  }
  for (int i = 0; i < rot / 2; ++i) {
    const double f = pow(base, -2.0 * i / rot);
    double slow = 0.0;                                    // the share of the slowed frequency
    if (scaling == BPDQ_ROTARY_LINEAR) slow = 1.0;
    if (scaling == BPDQ_ROTARY_YARN) slow = (i - ramp_lo) / (ramp_hi - ramp_lo);
    if (scaling == BPDQ_ROTARY_BANDS) slow = (high - original * f / two_pi) / (high - low);
    slow = fmin(fmax(slow, 0.0), 1.0);
    freq[i] = scaling == BPDQ_ROTARY_PLAIN || scaling == BPDQ_ROTARY_NTK ? f : f / factor * slow + f * (1.0 - slow);
  }
  if (mscale) *mscale = scaling == BPDQ_ROTARY_YARN ? 0.1 * log(factor) + 1.0 : 1.0;
  return 0;
}

extern "C" int bpdq_rotary(const double* freq, int rot, int layout, float mscale, int inverse, const int* pos, const int* tok_start,
                           int n_seq, int n_tok, int max_tok, const void* Q, long ldq, int n_q, const void* K, long ldk, int n_kv,
                           int head_dim, int dtype, void* Q_out, long ldqo, void* K_out, long ldko, void* stream_) {
  if (head_dim <= 0 || head_dim > kRotDimMost) return -17;
  if (rot <= 0 || rot % 2 || rot > head_dim) return -2;
  if (layout != BPDQ_ROTARY_HALF && layout != BPDQ_ROTARY_INTERLEAVED) return -3;
  if (!(mscale - mscale == 0.f)) return -4;
  if (n_seq < 0 || n_seq > 65535) return -8;
  if (n_tok < 0) return -9;
  if (max_tok < 0) return -10;
  if (n_q < 0 || n_q > 65535) return -13;
  if (n_kv < 0 || n_kv > 65535) return -16;
  if (dtype != BPDQ_F32 && dtype != BPDQ_F16 && dtype != BPDQ_BF16) return -18;
  if (n_seq == 0 || n_tok == 0 || max_tok == 0 || n_q + n_kv == 0) return 0;
  const size_t size = dtype == BPDQ_F32 ? 4 : 2;
  const long row_q = (long)n_q * head_dim, row_k = (long)n_kv * head_dim;
  auto bad = [&](const void* p, int heads) { return heads > 0 && (!p || reinterpret_cast<uintptr_t>(p) % size); };
  if (!freq || (reinterpret_cast<uintptr_t>(freq) & 7)) return -1;
  if (!pos || (reinterpret_cast<uintptr_t>(pos) & 3)) return -6;
  if (!tok_start || (reinterpret_cast<uintptr_t>(tok_start) & 3)) return -7;
  if (bad(Q, n_q)) return -11;
  if (ldq < row_q) return -12;
  if (bad(K, n_kv)) return -14;
  if (ldk < row_k) return -15;
  if (bad(Q_out, n_q)) return -19;
  if (ldqo < row_q || (Q_out == Q && ldqo != ldq)) return -20;
  if (bad(K_out, n_kv)) return -21;
  if (ldko < row_k || (K_out == K && ldko != ldk)) return -22;
  RotaryArgs a;
  a.freq = freq;
  a.pos = pos;
  a.tok_start = tok_start;
  a.q = Q;
  a.k = K;
  a.q_out = Q_out;
  a.k_out = K_out;
  a.ldq = ldq;
  a.ldk = ldk;
  a.ldqo = ldqo;
  a.ldko = ldko;
  a.rot = rot;
  a.half = layout == BPDQ_ROTARY_HALF;
  a.n_tok = n_tok;
  a.max_tok = max_tok < n_tok ? max_tok : n_tok;          // a sequence has no more rows than there are
  a.n_q = n_q;
  a.n_kv = n_kv;
  a.dim = head_dim;
  a.copy_q = Q_out != Q;
  a.copy_k = K_out != K;
  a.mscale = mscale;
  a.sign = inverse ? -1.f : 1.f;
  a.per = kRotPer;
  if ((long)bpdq_ceil_div(a.max_tok, kRotPer) * n_seq < 1024) a.per = 1;
  if ((long)bpdq_ceil_div(a.max_tok, a.per) * kRotThreads > 0xffffffffL) return -10;           // threads along the grid's x
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (dtype == BPDQ_F32) return rotary_launch<float>(a, n_seq, stream);
  if (dtype == BPDQ_F16) return rotary_launch<_Float16>(a, n_seq, stream);
  return rotary_launch<__bf16>(a, n_seq, stream);
}
