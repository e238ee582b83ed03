// rope_kernels.hip -- rotary positions of Q and K (seer_rope) and the append of new
// keys and values to a paged cache (seer_kv_append).
//
// Both move memory: two reads or writes of every element and some 20 operations on
// it.  A thread owns 16 planes' halves of one token (two 16-byte pieces of a head in
// bf16, 8 planes in fp32: VEC planes each), forms their cosines and sines once and
// walks over heads with them, so that the angles (about 30 instructions a plane) are shared by
// up to HB heads and every access is 16 bytes.  No table of cosines is read: the angle is an
// integer product of the position and the plane's turn rate (decode.h).
#include <algorithm>

#include "decode.h"

namespace seer {

namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;  // heads whose loads are in flight together

template <typename T>
struct Vec;
template <>
struct Vec<uint16_t> {  // bf16
  static constexpr int N = 8;
  using Raw = u32x4;
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(r[i] << 16);
      x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Raw pack(const float (&x)[8]) {
    union {
      bf16x8 v;
      Raw r;
    } u;
#pragma unroll
    for (int i = 0; i < 8; ++i) u.v[i] = (__bf16)x[i];
    return u.r;
  }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  using Raw = u32x4;
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(r[i]);
  }
  static __device__ __forceinline__ Raw pack(const float (&x)[4]) {
    Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(x[i]);
    return r;
  }
};

// A thread's two 16-byte pieces of a head: where they begin, and whether they turn.
template <typename T>
struct Pieces {
  int lo, hi;
  bool turn;
};
template <typename T, int D, bool INTER>
__device__ __forceinline__ Pieces<T> pieces(int c, int rot) {
  constexpr int N = Vec<T>::N;
  Pieces<T> p;
  p.turn = c < rot / (2 * N);
  if (p.turn && !INTER) {
    p.lo = c * N;
    p.hi = rot / 2 + c * N;
  } else {  // adjacent planes, or elements past rot: 2N elements in a row
    p.lo = 2 * c * N;
    p.hi = p.lo + N;
  }
  return p;
}

// The factors of the thread's N planes at position pos (scale in both).
template <int N>
__device__ __forceinline__ void factors(const RopeView& r, int c, int pos, bool grad, float (&cs)[N], float (&sn)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float co, si;
    turn_cos_sin(turn_rate(r.freq[c * N + i]), pos, co, si);
    cs[i] = co * r.scale;
    sn[i] = si * (grad ? -r.scale : r.scale);
  }
}

template <typename T, bool INTER>
__device__ __forceinline__ void turn(u32x4& lo, u32x4& hi, const float (&cs)[Vec<T>::N], const float (&sn)[Vec<T>::N]) {
  constexpr int N = Vec<T>::N;
  float a[N], b[N], x[N], y[N];
  Vec<T>::unpack(lo, a);
  Vec<T>::unpack(hi, b);
  if constexpr (INTER) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      x[2 * i] = a[2 * i] * cs[i] - a[2 * i + 1] * sn[i];
      x[2 * i + 1] = a[2 * i] * sn[i] + a[2 * i + 1] * cs[i];
      y[2 * i] = b[2 * i] * cs[N / 2 + i] - b[2 * i + 1] * sn[N / 2 + i];
      y[2 * i + 1] = b[2 * i] * sn[N / 2 + i] + b[2 * i + 1] * cs[N / 2 + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = a[i] * cs[i] - b[i] * sn[i];
      y[i] = a[i] * sn[i] + b[i] * cs[i];
    }
  }
  lo = Vec<T>::pack(x);
  hi = Vec<T>::pack(y);
}

template <typename T, int D, bool INTER>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a, FastDiv per_b, int hb) {
  constexpr int N = Vec<T>::N, TPT = D / (2 * N), TOK = kThreads / TPT;
  const int t = (int)blockIdx.x * TOK + (int)threadIdx.x / TPT;  // tokens of all batch entries in a row
  const int c = threadIdx.x % TPT;
  if (t >= a.batch * a.seq_len) return;
  const int b = fast_quot(per_b, t), s = t - b * a.seq_len;
  const Pieces<T> p = pieces<T, D, INTER>(c, a.rope.rot);
  float cs[N], sn[N];
  if (p.turn) {
    const int pos = a.positions ? a.positions[b * a.pos_stride + s] : a.start + s;
    factors<N>(a.rope, c, pos, a.grad, cs, sn);
  }
  const int heads = a.heads_q + a.heads_kv;
  const int h0 = blockIdx.y * hb, h1 = min(h0 + hb, heads);
  auto at = [&](const TensorView& t, int h) { return (T*)t.ptr + b * t.sb + h * t.sh + s * t.ss; };
  for (int h = h0; h < h1; h += kAhead) {
    u32x4 lo[kAhead], hi[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int g = min(h + i, h1 - 1);
      const T* src = g < a.heads_q ? at(a.q, g) : at(a.k, g - a.heads_q);
      lo[i] = *(const u32x4*)(src + p.lo);
      hi[i] = *(const u32x4*)(src + p.hi);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (h + i >= h1) break;
      T* dst = h + i < a.heads_q ? at(a.qo, h + i) : at(a.ko, h + i - a.heads_q);
      if (p.turn) turn<T, INTER>(lo[i], hi[i], cs, sn);
      *(u32x4*)(dst + p.lo) = lo[i];
      *(u32x4*)(dst + p.hi) = hi[i];
    }
  }
}

// A thread's planes of one token of every head of its share: K rotated, V copied.
template <typename T, int D, bool INTER>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, FastDiv per_b, int hb) {
  constexpr int N = Vec<T>::N, TPT = D / (2 * N), TOK = kThreads / TPT;
  const int t = (int)blockIdx.x * TOK + (int)threadIdx.x / TPT;  // tokens of all batch entries in a row
  const int c = threadIdx.x % TPT;
  if (t >= a.batch * a.tokens) return;
  const int b = fast_quot(per_b, t), s = t - b * a.tokens;
  const int pos = a.positions[b * a.pos_stride + s];
  const int row = a.rows ? a.rows[b * a.pos_stride + s] : b;
  if (pos < 0 || row < 0 || row >= a.table.rows) return;
  const int i = fast_quot(a.table.page, pos);
  if (i >= a.table.max_pages) return;
  const int page = a.table.ptr[row * a.table.stride + i];
  if (page < 0 || page >= a.table.num_pages) return;
  const int slot = pos - i * a.table.page.d;
  const Pieces<T> p = pieces<T, D, INTER>(c, a.rope.rot);
  float cs[N], sn[N];
  if (p.turn) factors<N>(a.rope, c, pos, false, cs, sn);
  const int h0 = blockIdx.y * hb, h1 = min(h0 + hb, a.heads_kv);
  const T* k = (const T*)a.k.ptr + b * a.k.sb + s * a.k.ss;
  const T* v = (const T*)a.v.ptr + b * a.v.sb + s * a.v.ss;
  T* kc = (T*)a.kc.ptr + page * a.kc.sp + slot * a.kc.ss;
  T* vc = (T*)a.vc.ptr + page * a.vc.sp + slot * a.vc.ss;
  constexpr int U = kAhead / 2;
  for (int h = h0; h < h1; h += U) {
    u32x4 klo[U], khi[U], vlo[U], vhi[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int g = min(h + j, h1 - 1);
      klo[j] = *(const u32x4*)(k + g * a.k.sh + p.lo);
      khi[j] = *(const u32x4*)(k + g * a.k.sh + p.hi);
      vlo[j] = *(const u32x4*)(v + g * a.v.sh + p.lo);
      vhi[j] = *(const u32x4*)(v + g * a.v.sh + p.hi);
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (h + j >= h1) break;
      if (p.turn) turn<T, INTER>(klo[j], khi[j], cs, sn);
      *(u32x4*)(kc + (h + j) * a.kc.sh + p.lo) = klo[j];
      *(u32x4*)(kc + (h + j) * a.kc.sh + p.hi) = khi[j];
      *(u32x4*)(vc + (h + j) * a.vc.sh + p.lo) = vlo[j];
      *(u32x4*)(vc + (h + j) * a.vc.sh + p.hi) = vhi[j];
    }
  }
}

// Heads per workgroup: as many as leave the launch 2048 workgroups, 1 to 8.
int head_share(int64_t tiles, int heads) {
  int hb = 8;
  while (hb > 1 && tiles * ((heads + hb - 1) / hb) < 2048) hb /= 2;
  return hb;
}

template <typename T, int D>
hipError_t rotate(const RotateArgs& a, hipStream_t s) {
  constexpr int TOK = kThreads / (D / (2 * Vec<T>::N));
  const int64_t tiles = ((int64_t)a.batch * a.seq_len + TOK - 1) / TOK;
  const int heads = a.heads_q + a.heads_kv;
  const int hb = head_share(tiles, heads);
  const dim3 grid((unsigned)tiles, (unsigned)((heads + hb - 1) / hb));
  if (a.rope.interleaved) rotate_kernel<T, D, true><<<grid, kThreads, 0, s>>>(a, fast_div(a.seq_len), hb);
  else rotate_kernel<T, D, false><<<grid, kThreads, 0, s>>>(a, fast_div(a.seq_len), hb);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  constexpr int TOK = kThreads / (D / (2 * Vec<T>::N));
  const int64_t tiles = ((int64_t)a.batch * a.tokens + TOK - 1) / TOK;
  const int hb = head_share(tiles, a.heads_kv);
  const dim3 grid((unsigned)tiles, (unsigned)((a.heads_kv + hb - 1) / hb));
  if (a.rope.interleaved) append_kernel<T, D, true><<<grid, kThreads, 0, s>>>(a, fast_div(a.tokens), hb);
  else append_kernel<T, D, false><<<grid, kThreads, 0, s>>>(a, fast_div(a.tokens), hb);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, hipStream_t s) {
  if (a.bf16) return a.head_dim == 128 ? rotate<uint16_t, 128>(a, s) : rotate<uint16_t, 64>(a, s);
  return a.head_dim == 128 ? rotate<float, 128>(a, s) : rotate<float, 64>(a, s);
}

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  if (a.bf16) return a.head_dim == 128 ? append<uint16_t, 128>(a, s) : append<uint16_t, 64>(a, s);
  return a.head_dim == 128 ? append<float, 128>(a, s) : append<float, 64>(a, s);
}

}  // namespace seer
