// decode.h -- internal launchers behind include/seer_decode.h, and the rotation that
// its kernels share.  Arguments are validated by the ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.h"
#include "launch.h"

namespace seer {

struct RopeView {
  const double* freq;  // nullptr: no rotation
  int rot;             // rotated elements of a head, a multiple of 16
  int interleaved;
  float scale;
};

// n / d for 0 <= n < 2^31 and a fixed d >= 1, by a multiplication (Granlund and
// Montgomery): n / d = (n + hi(m n)) >> s, m = floor(2^32 (2^s - d) / d) + 1, s = ceil(log2 d).
struct FastDiv {
  uint32_t m, s;
  int d;
};
inline FastDiv fast_div(int d) {
  FastDiv f;
  f.d = d;
  f.s = 0;
  while ((1ull << f.s) < (uint64_t)d) ++f.s;
  f.m = (uint32_t)((((1ull << f.s) - (uint64_t)d) << 32) / (uint64_t)d + 1);
  return f;
}

struct CacheView {  // pool of pages of one of K and V, element strides
  const void* ptr;
  int64_t sp, sh, ss;
};

struct PageTable {
  const int32_t* ptr;
  int64_t stride;
  int rows, max_pages, num_pages;
  FastDiv page;
};

struct RotateArgs {
  TensorView q, k, qo, ko;  // (output pointers are written)
  int batch, heads_q, heads_kv, seq_len, head_dim;
  bool bf16, grad;
  RopeView rope;
  const int32_t* positions;
  int64_t pos_stride;
  int start;
};

struct AppendArgs {
  TensorView k, v;
  CacheView kc, vc;
  PageTable table;
  int batch, tokens, heads_kv, head_dim;
  bool bf16;
  RopeView rope;
  const int32_t* positions;
  const int32_t* rows;
  int64_t pos_stride;
};

struct PagedArgs {
  TensorView q;
  void* o;
  int64_t osb, osh, oss;
  float* lse;
  CacheView kc, vc;
  PageTable table;
  const int32_t* positions;
  int64_t pos_stride;
  int batch, heads_q, heads_kv, tokens, head_dim;
  bool bf16;
  RopeView rope;
  float scale;
  void* workspace;
};

hipError_t launch_rotate(const RotateArgs& a, hipStream_t s);
hipError_t launch_append(const AppendArgs& a, hipStream_t s);
hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t s);
size_t paged_attn_workspace(int batch, int heads_q, int heads_kv, int tokens, int head_dim);

#ifdef __HIPCC__
__device__ __forceinline__ int fast_quot(const FastDiv& f, int n) {
  return (int)((__umulhi((uint32_t)n, f.m) + (uint32_t)n) >> f.s);
}

// A plane's angle per position as a fraction of a turn in 64-bit fixed point, within 2^-64 of a turn and 2^-52 of itself:
// position times it, modulo 2^64, is the angle modulo a turn with no further rounding.
struct TurnRate {
  uint32_t hi, lo;
};
__device__ __forceinline__ TurnRate turn_rate(double inv_freq) {
  double t = inv_freq * 0.15915494309189533577;  // 1 / (2 pi)
  t -= trunc(t);
  const double u = fabs(t) * 4294967296.0;
  const uint32_t hi = (uint32_t)u;
  uint64_t r = (uint64_t)hi << 32 | (uint32_t)((u - (double)hi) * 4294967296.0);
  if (t < 0) r = 0 - r;  // (backwards: the magnitude first, as 1 + t would round small ones away)
  return {(uint32_t)(r >> 32), (uint32_t)r};
}

// cos and sin of pos * rate, to fp32 rounding: the fraction of a turn less its nearest
// quarter, at most pi / 4 off it, where the Taylor series to x^9 and x^8 are within 3e-8.  The low word counts where the
// rest is small: a slow plane near position 0 (2.5e-6 per position) has a sine 0.05% off without it.
__device__ __forceinline__ void turn_cos_sin(const TurnRate& r, int pos, float& c, float& s) {
  const uint32_t lo = (uint32_t)pos * r.lo;
  uint32_t x = (uint32_t)pos * r.hi + __umulhi((uint32_t)pos, r.lo);
  if (pos < 0) x -= r.lo;  // (the unsigned product is 2^32 rate too large)
  x += lo >> 31;           // the high word to nearest, the low one signed
  const uint32_t quarter = (x + 0x20000000u) >> 30;
  // 2 pi 2^-64 and 2 pi 2^-32
  const float y = fmaf((float)(int32_t)lo, 3.40612158e-19f, (float)(int32_t)(x - (quarter << 30)) * 1.46291807926715968e-9f);
  const float y2 = y * y;
  float sn = fmaf(y2, 2.7557319e-6f, -1.98412698e-4f);
  sn = fmaf(y2, sn, 8.33333333e-3f);
  sn = fmaf(y2, sn, -1.66666667e-1f);
  sn = fmaf(y2 * y, sn, y);
  float cn = fmaf(y2, 2.48015873e-5f, -1.38888889e-3f);
  cn = fmaf(y2, cn, 4.16666667e-2f);
  cn = fmaf(y2, cn, -0.5f);
  cn = fmaf(y2, cn, 1.0f);
  const float a = (quarter & 1) ? sn : cn, b = (quarter & 1) ? cn : sn;
  c = (quarter + 1) & 2 ? -a : a;
  s = quarter & 2 ? -b : b;
}
#endif

}  // namespace seer
