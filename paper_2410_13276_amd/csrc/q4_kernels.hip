// q4_kernels.hip -- tokens into a paged cache held in 4 bits (seer_kv_append_q4), and out of a cache of either
// kind (seer_kv_read).
//
// Both move memory.  A thread owns 8 elements of a head: 16 bytes of bf16 (32 of fp32) against one
// dword of codes, so that a wavefront's accesses to values are whole lines and those to codes 64-byte runs; 4 or 8 neighbours hold a
// group and find its range by exchanges within a row of lanes.  A thread walks over its token's heads, so that pages
// and angles are found once for them.
//
// A code is floor((x - middle) / step) + 8, decided exactly: fp32 gives the quotient to within 1e-5, and where that is
// nearer to a whole number b than this, the sign of x - middle - b step decides, which three fp32 operations give without
// error (x - middle as a sum of two numbers, b step exact: 4 by 8 bits).
//
// 25000 tokens of 8 heads of 128 in groups of 32 (bf16, 135 MB), one MI355X: stored in 34 us, bound by its vector instructions (18.8e6
// of wavefronts, 31 us of issue; the memory would take 27), rotated in 39; read in 23.5, 5.7e12 bytes a second, as a copy's.
#include <algorithm>

#include "cache.h"
#include "paged_common.h"

namespace seer {

namespace {

constexpr int kThreads = 256;
// loads of values that a thread has in flight: 2 K and 2 V heads stored, 2 and 2 read (with 4 and 4, 25000 tokens of 8 heads of 128:
// stored 31 -> 34 us, read 22.8 -> 23.0, of 4 heads of 64 7.1 -> 7.7)
constexpr int kAhead = 4;
constexpr int kReadAhead = 2;

template <typename T>
struct Eight;  // 8 elements as a thread moves them
template <>
struct Eight<uint16_t> {
  using Raw = u32x4[1];
  static __device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
    union {
      bf16x8 v;
      u32x4 r;
    } u;
#pragma unroll
    for (int i = 0; i < 8; ++i) u.v[i] = (__bf16)x[i];
    return u.r;
  }
};
template <>
struct Eight<float> {
  using Raw = u32x4[2];
};
template <typename T>
__device__ __forceinline__ void load8(const T* p, typename Eight<T>::Raw& r) {
  r[0] = *(const u32x4*)p;
  if constexpr (sizeof(T) == 4) r[1] = *(const u32x4*)(p + 4);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    __builtin_nontemporal_store(Eight<T>::pack(x), (u32x4*)p);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *((u32x4*)p + i) = u32x4{__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]),
                               __float_as_uint(x[4 * i + 3])};
  }
}

// Largest of the LANES (4 or 8) neighbours, for all of them.
template <int LANES>
__device__ __forceinline__ float neighbours_max(float x) {
  auto with = [&](int y) { x = fmaxf(x, __int_as_float(y)); };
  with(dpp<0xb1>(0, __float_as_int(x)));  // quad_perm 1 0 3 2
  with(dpp<0x4e>(0, __float_as_int(x)));  // quad_perm 2 3 0 1
  if constexpr (LANES == 8) with(dpp<0x141>(0, __float_as_int(x)));  // row_half_mirror
  return x;
}

struct Held {
  uint32_t codes, params;
};

// a - b as d + e exactly.
struct Two {
  float d, e;
};
__device__ __forceinline__ Two exact_difference(float a, float b) {
  const float d = a - b, back = d - a;
  return {d, (a - (d - back)) - (b + back)};
}

// 8 elements of a group that LANES neighbours hold.
template <int LANES>
__device__ __forceinline__ Held hold(const float (&x)[8]) {
  // (maximum and minimum are NaN where an element is)
  float hi = x[0], lo = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    hi = __builtin_elementwise_maximum(hi, x[i]);
    lo = __builtin_elementwise_minimum(lo, x[i]);
  }
  hi = neighbours_max<LANES>(hi <= 0x1p127f && lo >= -0x1p127f ? hi : INFINITY);
  lo = -neighbours_max<LANES>(-lo);
  if (hi == INFINITY) return {0x88888888u, 0x7fc0u};  // step NaN, middle 0
  const float mid = (float)(__bf16)(0.5f * hi + 0.5f * lo);
  // the step: the first of three numbers, from the fp32 quotient without its low bits on, from which 7.5 steps reach
  // (7.5 of them are exact, and so is the difference from what they are compared with, which is near)
  const Two up = exact_difference(hi, mid), down = exact_difference(mid, lo);
  const bool lower = down.d > up.d || (down.d == up.d && down.e > up.e);
  const float reach = lower ? down.d : up.d, rest = lower ? down.e : up.e;
  uint32_t step = __float_as_uint(reach * (1.f / 7.5f)) & 0xffff0000u;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if ((7.5f * __uint_as_float(step) - reach) - rest < 0.f) step += 0x10000u;
  step = reach > 0.f ? max(step, 0x0d800000u) : 0u;  // 2^-100
  const float s = __uint_as_float(step);
  const float inv = step ? __builtin_amdgcn_rcpf(s) : 0.f;
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = x[i] - mid;
    const float y = fmaf(d, inv, 8.f), b = rintf(y);  // (within 0.5 to 15.5, but for rounding)
    float f = y;
    if (fabsf(y - b) < 1e-5f) {
      const Two z = exact_difference(x[i], mid);
      f = (z.d - (b - 8.f) * s) + z.e >= 0.f ? b : b - 1.f;
    }
    codes |= (uint32_t)f << 4 * i;
  }
  return {codes, step >> 16 | (__float_as_uint(mid) & 0xffff0000u)};
}

// Where a token of the call stands; false: padding, or no page.
struct Place {
  int b, s, page, slot;
  int64_t at;  // of positions
};
__device__ __forceinline__ bool place_of(const StoreArgs& a, const FastDiv& per_b, int t, Place& p) {
  p.b = fast_quot(per_b, t);
  p.s = t - p.b * a.tokens;
  p.at = p.b * a.pos_stride + p.s;
  const PageTable& tab = a.cache.table;
  const int pos = a.positions[p.at];
  const int row = a.rows ? a.rows[p.at] : p.b;
  if (pos < 0 || row < 0 || row >= tab.rows) return false;
  const int i = fast_quot(tab.page, pos);
  if (i >= tab.max_pages) return false;
  p.page = tab.ptr[row * tab.stride + i];
  p.slot = pos - i * tab.page.d;
  return p.page >= 0 && p.page < tab.num_pages;
}

template <typename T, int D, int GROUP, int ROPE>  // ROPE 0: none, 1: halves, 2: adjacent elements
__global__ __launch_bounds__(kThreads) void append_q4_kernel(StoreArgs a, FastDiv per_b, int hb) {
  constexpr int TPT = D / 8, TOK = kThreads / TPT, LANES = GROUP / 8;
  const int t = (int)blockIdx.x * TOK + (int)threadIdx.x / TPT;
  const int c = threadIdx.x % TPT, d0 = 8 * c;
  if (t >= a.batch * a.tokens) return;
  Place p;
  if (!place_of(a, per_b, t, p)) return;
  // cosines and sines of the piece's planes, and where their other elements stand
  const bool turns = ROPE != 0 && d0 < a.rope.rot;
  const int half = a.rope.rot / 2;
  const bool second = ROPE == 1 && d0 >= half;
  const int other = turns && ROPE == 1 ? (second ? d0 - half : d0 + half) : d0;
  float2 cs[ROPE == 1 ? 8 : 4];
  if (turns) {
    const int pos = a.rope_positions[p.at];
    const int plane = ROPE == 1 ? (second ? d0 - half : d0) : d0 / 2;
#pragma unroll
    for (int i = 0; i < (ROPE == 1 ? 8 : 4); ++i) {
      float co, si;
      turn_cos_sin(turn_rate(a.rope.freq[plane + i]), pos, co, si);
      cs[i] = make_float2(co * a.rope.scale, si * a.rope.scale);
    }
  }
  const int h0 = blockIdx.y * hb, h1 = min(h0 + hb, a.cache.heads_kv);
  const T* k = (const T*)a.k.ptr + p.b * a.k.sb + p.s * a.k.ss;
  const T* v = (const T*)a.v.ptr + p.b * a.v.sb + p.s * a.v.ss;
  auto put = [&](const PoolView& pool, int h, const Held& x) {
    *(uint32_t*)((char*)pool.data + p.page * pool.sp + h * pool.sh + p.slot * pool.ss + 4 * c) = x.codes;
    if (c % LANES == 0)
      ((uint32_t*)pool.params)[p.page * pool.psp + h * pool.psh + p.slot * pool.pss + c / LANES] = x.params;
  };
  constexpr int U = kAhead / 2;
  for (int h = h0; h < h1; h += U) {
    typename Eight<T>::Raw kr[U], ko[U], vr[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int g = min(h + j, h1 - 1);
      load8(k + g * a.k.sh + d0, kr[j]);
      if (ROPE == 1) load8(k + g * a.k.sh + other, ko[j]);
      load8(v + g * a.v.sh + d0, vr[j]);
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (h + j >= h1) break;
      float y[8], z[8];
      unpack8(kr[j], y);
      if constexpr (ROPE == 1) {
        unpack8(ko[j], z);
        if (turns)
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = y[i] * cs[i].x + z[i] * (second ? cs[i].y : -cs[i].y);
      } else if constexpr (ROPE == 2) {
        if (turns)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float u = y[2 * i], w = y[2 * i + 1];
            y[2 * i] = u * cs[i].x - w * cs[i].y;
            y[2 * i + 1] = u * cs[i].y + w * cs[i].x;
          }
      }
      put(a.cache.k, h + j, hold<LANES>(y));
      unpack8(vr[j], y);
      put(a.cache.v, h + j, hold<LANES>(y));
    }
  }
}

// GROUP 0: the values are moved as they are.
template <typename T, int D, int GROUP>
__global__ __launch_bounds__(kThreads) void read_kernel(StoreArgs a, FastDiv per_b, int hb) {
  constexpr int TPT = D / 8, TOK = kThreads / TPT;
  const int t = (int)blockIdx.x * TOK + (int)threadIdx.x / TPT;
  const int c = threadIdx.x % TPT;
  if (t >= a.batch * a.tokens) return;
  Place p;
  const bool there = place_of(a, per_b, t, p);
  if (!there) p.page = p.slot = 0;
  const int h0 = blockIdx.y * hb, h1 = min(h0 + hb, a.cache.heads_kv);
  for (int h = h0; h < h1; h += kReadAhead) {
    uint32_t codes[2][kReadAhead], params[2][kReadAhead];
    typename Eight<T>::Raw raw[2][kReadAhead];
#pragma unroll
    for (int j = 0; j < kReadAhead; ++j) {
      const int g = min(h + j, h1 - 1);
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const PoolView& pool = f ? a.cache.v : a.cache.k;
        const int64_t off = p.page * pool.sp + g * pool.sh + p.slot * pool.ss;
        if constexpr (GROUP == 0) {
          load8((const T*)pool.data + off + 8 * c, raw[f][j]);
        } else {
          codes[f][j] = *(const uint32_t*)((const char*)pool.data + off + 4 * c);
          params[f][j] = pool.params[p.page * pool.psp + g * pool.psh + p.slot * pool.pss + 8 * c / GROUP];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kReadAhead; ++j) {
      if (h + j >= h1) break;
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const TensorView& out = f ? a.v : a.k;
        float x[8];
        if constexpr (GROUP == 0) {
          unpack8(raw[f][j], x);
        } else {
          const float step = __uint_as_float(params[f][j] << 16), mid = __uint_as_float(params[f][j] & 0xffff0000u);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = fmaf((float)(codes[f][j] >> 4 * i & 15u) - 7.5f, step, mid);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = there ? x[i] : 0.f;
        store8((T*)out.ptr + p.b * out.sb + (h + j) * out.sh + p.s * out.ss + 8 * c, x);
      }
    }
  }
}

// Heads per workgroup, whose threads find their token's place and angles once for all of them: at most `most`, fewer where that leaves
// the launch less than 1024 workgroups (with 2048, 2000 tokens of 32 heads of 128 are stored in 14.2 instead of 13.1 us, rotated in 24.0
// instead of 17.9, read in 11.2 instead of 9.6).
int head_share(int64_t tiles, int heads, int most) {
  int hb = most;
  while (hb > 1 && tiles * ((heads + hb - 1) / hb) < 1024) hb /= 2;
  return hb;
}

struct Grid {
  dim3 grid;
  FastDiv per_b;
  int hb;
};
Grid grid_of(const StoreArgs& a) {
  const int tok = kThreads / (a.cache.head_dim / 8);
  const int64_t tiles = ((int64_t)a.batch * a.tokens + tok - 1) / tok;
  // (rotated 8: 20000 tokens of 32 heads 104 us, with 4 112; else 4: 25000 tokens of 8 heads 31.2 us, with 8 33.6)
  const int hb = head_share(tiles, a.cache.heads_kv, a.rope.freq ? 8 : 4);
  return {dim3((unsigned)tiles, (unsigned)((a.cache.heads_kv + hb - 1) / hb)), fast_div(a.tokens), hb};
}

template <typename T, int D, int GROUP>
hipError_t append(const StoreArgs& a, hipStream_t s) {
  const Grid g = grid_of(a);
  if (!a.rope.freq) append_q4_kernel<T, D, GROUP, 0><<<g.grid, kThreads, 0, s>>>(a, g.per_b, g.hb);
  else if (a.rope.interleaved) append_q4_kernel<T, D, GROUP, 2><<<g.grid, kThreads, 0, s>>>(a, g.per_b, g.hb);
  else append_q4_kernel<T, D, GROUP, 1><<<g.grid, kThreads, 0, s>>>(a, g.per_b, g.hb);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t append(const StoreArgs& a, hipStream_t s) {
  return a.cache.group == 64 ? append<T, D, 64>(a, s) : append<T, D, 32>(a, s);
}

template <typename T, int D>
hipError_t read(const StoreArgs& a, hipStream_t s) {
  const Grid g = grid_of(a);
  if (a.cache.group == 64) read_kernel<T, D, 64><<<g.grid, kThreads, 0, s>>>(a, g.per_b, g.hb);
  else if (a.cache.group == 32) read_kernel<T, D, 32><<<g.grid, kThreads, 0, s>>>(a, g.per_b, g.hb);
  else read_kernel<T, D, 0><<<g.grid, kThreads, 0, s>>>(a, g.per_b, g.hb);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append_q4(const StoreArgs& a, hipStream_t s) {
  if (a.bf16) return a.cache.head_dim == 128 ? append<uint16_t, 128>(a, s) : append<uint16_t, 64>(a, s);
  return a.cache.head_dim == 128 ? append<float, 128>(a, s) : append<float, 64>(a, s);
}

hipError_t launch_read(const StoreArgs& a, hipStream_t s) {
  if (a.bf16) return a.cache.head_dim == 128 ? read<uint16_t, 128>(a, s) : read<uint16_t, 64>(a, s);
  return a.cache.head_dim == 128 ? read<float, 128>(a, s) : read<float, 64>(a, s);
}

}  // namespace seer
