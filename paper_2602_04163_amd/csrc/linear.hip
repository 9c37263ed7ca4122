// The C entry of the product on stored planes (linear.h): checks, and the unit of the number of planes.
#include "linear.h"

using namespace bpdq;

extern "C" size_t bpdq_linear_workspace_bytes(int n_tok, int d_in) {
  if (n_tok <= kLinRowsMost || d_in <= 0 || d_in % 32) return 0;
  return linear_image_bytes(n_tok, d_in) + bpdq_align_up((size_t)n_tok, kLinTokPad) * sizeof(uint32_t);
}

extern "C" int bpdq_linear(const uint32_t* planes, const uint16_t* coefs_h, int d_out, int d_in, int bits, int group,
                           const void* X, int n_tok, long ldx, int dtype, const void* bias, int act, const void* residual,
                           long ldr, void* Y, long ldy, void* ws, size_t ws_bytes, void* stream_) {
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
  const size_t need = bpdq_linear_workspace_bytes(n_tok, d_in);
  if (need && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255))) return -17;
  if (ws_bytes < need) return -18;
  LinearArgs a;
  a.planes = planes;
  a.coefs = reinterpret_cast<const _Float16*>(coefs_h);
  a.x = X;
  a.bias = bias;
  a.residual = residual;
  a.y = Y;
  a.ws = ws;
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
  a.vec_y = reinterpret_cast<uintptr_t>(Y) % 16 == 0 && ldy % 8 == 0;
  a.vec_r = reinterpret_cast<uintptr_t>(residual) % 16 == 0 && ldr % 8 == 0;
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  switch (bits) {
    case 1: return linear_run<1>(a, dtype, stream);
    case 2: return linear_run<2>(a, dtype, stream);
    case 3: return linear_run<3>(a, dtype, stream);
    default: return linear_run<4>(a, dtype, stream);
  }
}
