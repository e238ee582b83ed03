// q4_open.h -- codes of 4 bits as operands of a matrix product.
#pragma once

#include "cache.h"
#include "paged_common.h"

namespace seer {

// 1 + c / 16 for c = 7.5, halfway between the codes
constexpr float kMid = 1.46875f;

#ifdef __HIPCC__
// The 8 codes of a dword as bf16 1 + c / 16 in the order 0 4 1 5 2 6 3 7, codes 4 to 7 complemented.
__device__ __forceinline__ bf16x8 open8(uint32_t w) {
  u32x4 y;
  y[0] = (w << 3 & 0x00780078u) ^ 0x3ff83f80u;
  y[1] = (w >> 1 & 0x00780078u) ^ 0x3ff83f80u;
  y[2] = (w >> 5 & 0x00780078u) ^ 0x3ff83f80u;
  y[3] = (w >> 9 & 0x00780078u) ^ 0x3ff83f80u;
  return __builtin_bit_cast(bf16x8, y);
}

// The same codes as (c - 7.5) / 16, in the same order and with the same ones complemented: for results in fp32, whose sums would
// carry the rounding of numbers 3 to 7 times the values'.  Sign and size of a code are its upper bit and the lower three, turned over
// below the middle; the bytes of the 8 sizes are looked up, four codes at a time.
__device__ __forceinline__ bf16x8 open8_centred(uint32_t w) {
  w ^= 0xffff0000u;
  u32x4 y;
#pragma unroll
  for (int odd = 0; odd < 2; ++odd) {
    const uint32_t c = odd ? w >> 4 : w;
    const uint32_t below = ~c & 0x08080808u;
    const uint32_t size = (c ^ (below - (below >> 3))) & 0x07070707u;
    const uint32_t lo = __builtin_amdgcn_perm(0xf0d0b090u, 0x6020c000u, size);
    const uint32_t hi = __builtin_amdgcn_perm(0x3e3e3e3eu, 0x3e3e3d3du, size) | below << 4;
    y[odd] = __builtin_amdgcn_perm(hi, lo, 0x06020400u);      // codes 0 and 4, 1 and 5
    y[odd + 2] = __builtin_amdgcn_perm(hi, lo, 0x07030501u);  // 2 and 6, 3 and 7
  }
  return __builtin_bit_cast(bf16x8, y);
}

// x as the sum of N bf16 parts: three hold fp32 exactly (8 significant bits each time); two, each rounded to nearest, are
// 2^-18 off at most.
template <int N>
__device__ __forceinline__ void split(const float (&x)[8], bf16x8 (&y)[N]) {
  if constexpr (N == 3) {
    split3(x, y);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[0][e] = (__bf16)x[e];
    if constexpr (N == 2)
#pragma unroll
      for (int e = 0; e < 8; ++e) y[1][e] = (__bf16)(x[e] - (float)y[0][e]);
  }
}

// A quarter of a key's codes of each of the four rows of 16 lanes (row j: quarter j) as operands whose 32 channels are
// successive: dword 4 f + j of the key to row j of operand f, by exchanges of rows between two registers.
template <int N>
__device__ __forceinline__ void by_channels(uint32_t (&x)[N]) {
  static_assert(N == 2 || N == 4, "dwords of a quarter");
  auto swap16 = [](uint32_t& a, uint32_t& b) {  // odd rows of a, even ones of b
    const auto y = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = y[0], b = y[1];
  };
  auto swap32 = [](uint32_t& a, uint32_t& b) {  // the upper half of a, the lower one of b
    const auto y = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = y[0], b = y[1];
  };
  swap16(x[0], x[1]);
  if constexpr (N == 4) {
    swap16(x[2], x[3]);
    swap32(x[0], x[2]);
    swap32(x[1], x[3]);
  } else {
    swap32(x[0], x[1]);
  }
}

// The share of workgroup `id` of `workers`.  Where pages are token-major, heads' codes share lines; with some sequences, successive
// shares go to one XCD then (workgroups go round the 8 XCDs), so that a sequence's heads meet in its L2.  Token-major, 32 / 8 heads of
// 128: 64 sequences of 3000 tokens attention 118 -> 77 us, weights 60 -> 49, 8 of 16000 56 -> 55 and 46 -> 39.5, 4 of 3000 (4 tokens each) 33 ->
// 28; one sequence of 131072 72 -> 86 and 32 -> 50 (its heads' shares lie apart by multiples of 8 anyhow).  Head-major, 28 rows of 4 heads over 8 x 4096
// tokens 35 -> 40.
__device__ __forceinline__ int share_of(const PoolView& k, int batch, int id, int workers) {
  if (k.sh >= k.ss || batch < 4) return id;
  const int xcd = id % 8, each = workers / 8;
  return xcd * each + min(xcd, workers % 8) + id / 8;
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(dpp<CTRL>(0, __float_as_int(x)));
}
#endif

}  // namespace seer
