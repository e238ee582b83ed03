// paged_common.h -- what the kernels that read a paged cache share: how work is dealt to workgroups,
// sums and maxima within a wavefront, and the query rows' rotation and split.
#pragma once

#include "decode.h"

namespace seer {

constexpr float kLn2 = 0.6931471805599453f;

struct Stride16 {
  uint32_t page, slot;
};

#ifdef __HIPCC__
// Where the page of the last of a run's keys [.., k_hi) stands in its table row, which look-ups of keys behind the run are
// held to.  A run without keys is held to the first entry: the quotient of -1 is a large number (pages of 16: 268435455).
__host__ __device__ __forceinline__ int last_page_of(const FastDiv& page, int k_hi) {
  return fast_quot(page, k_hi > 0 ? k_hi - 1 : 0);
}

// The weights dealt to the workgroups: workgroup w has base (+ 1 for the first `rest`).  (All below 2^30: the
// 64-bit divisions that this was first written with were 600 instructions at every workgroup's start.)
struct Deal {
  uint32_t base, rest, workers;
  __device__ __forceinline__ Deal(uint32_t total, uint32_t groups) {
    workers = min(groups, total);
    base = total / workers;
    rest = total - base * workers;
  }
  __device__ __forceinline__ int first(uint32_t w) const { return (int)(w * base + min(w, rest)); }
  __device__ __forceinline__ int owner(uint32_t x) const {
    const uint32_t big = rest * (base + 1);
    return (int)(x < big ? x / (base + 1) : rest + (x - big) / base);
  }
};

// Within a wavefront, without the LDS: inclusive prefix sum; least of a row of 16 lanes; largest and sum of the
// lanes l % 16.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int dpp(int old, int x) {
  return __builtin_amdgcn_update_dpp(old, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_prefix(int x) {
  x += dpp<0x111>(0, x);  // row_shr 1, 2, 4, 8
  x += dpp<0x112>(0, x);
  x += dpp<0x114>(0, x);
  x += dpp<0x118>(0, x);
  x += dpp<0x142, 0xa>(0, x);  // row_bcast 15 to rows 1 and 3
  x += dpp<0x143, 0xc>(0, x);  // row_bcast 31 to rows 2 and 3
  return x;
}
__device__ __forceinline__ int row_min(int x) {
  x = min(x, dpp<0xb1>(x, x));   // quad_perm 1 0 3 2
  x = min(x, dpp<0x4e>(x, x));   // quad_perm 2 3 0 1
  x = min(x, dpp<0x141>(x, x));  // row_half_mirror
  return min(x, dpp<0x140>(x, x));  // row_mirror
}
typedef __attribute__((ext_vector_type(2))) unsigned int u32pair;
__device__ __forceinline__ void across(float x, bool half, float& y, float& z) {
  const uint32_t u = __float_as_uint(x);
  const u32pair p = half ? __builtin_bit_cast(u32pair, __builtin_amdgcn_permlane32_swap(u, u, false, false))
                         : __builtin_bit_cast(u32pair, __builtin_amdgcn_permlane16_swap(u, u, false, false));
  y = __uint_as_float(p[0]);
  z = __uint_as_float(p[1]);
}
__device__ __forceinline__ float column_max(float x) {
  float y, z;
  across(x, false, y, z);
  x = fmaxf(y, z);
  across(x, true, y, z);
  return fmaxf(y, z);
}
__device__ __forceinline__ float column_sum(float x) {
  float y, z;
  across(x, false, y, z);
  x = y + z;
  across(x, true, y, z);
  return y + z;
}

__device__ __forceinline__ void unpack8(const u32x4 (&q)[1], float (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __uint_as_float(q[0][i] << 16);
    y[2 * i + 1] = __uint_as_float(q[0][i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack8(const u32x4 (&q)[2], float (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(q[i / 4][i % 4]);
}

// Elements d0 .. d0 + 7 of a head, y, rotated; z: the other half of their planes (half layout), cs: cosine and sine of the
// token's planes.
__device__ __forceinline__ void rotate8(const RopeView& r, const float2* cs, int d0, float (&y)[8], const float (&z)[8]) {
  if (r.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = cs[d0 / 2 + i];
      const float u = y[2 * i], v = y[2 * i + 1];
      y[2 * i] = u * f.x - v * f.y;
      y[2 * i + 1] = u * f.y + v * f.x;
    }
  } else {
    const bool second = d0 >= r.rot / 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = cs[(second ? d0 - r.rot / 2 : d0) + i];
      y[i] = y[i] * f.x + z[i] * (second ? f.y : -f.y);
    }
  }
}

// x as the sum of three bf16 parts, exactly: 8 significant bits of what is left each time.
__device__ __forceinline__ void split3(const float (&x)[8], bf16x8 (&y)[3]) {
  u32x4 z[3];
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
  for (int part = 0; part < 3; ++part) {
#pragma unroll
    for (int f = 0; f < 4; ++f)
      z[part][f] = __builtin_amdgcn_perm(__float_as_uint(rest[2 * f + 1]), __float_as_uint(rest[2 * f]), 0x07060302u);
#pragma unroll
    for (int e = 0; e < 8; ++e) rest[e] -= __uint_as_float(__float_as_uint(rest[e]) & 0xffff0000u);
    y[part] = __builtin_bit_cast(bf16x8, z[part]);
  }
}
#endif

}  // namespace seer
