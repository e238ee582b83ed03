// rope_kernels.hip -- rotary positions of Q and K (seer_rope) and the append of new
// keys and values to a paged cache (seer_kv_append).
//
// Both move memory: a read and a write of every element, and some 10 operations on
// it.  A thread owns two 16-byte pieces of one token's heads (8 planes in bf16, 4 in fp32), forms their
// cosines and sines once and walks over up to 8 heads with them, so that the angles (about 50
// instructions a plane, its rate's among them) are shared and every access is 16 bytes.  No table of cosines is read: the angle is an
// integer product of the position and the plane's turn rate (decode.h).  Large calls run at a copy's rate (5.1 TB/s of
// reads and writes): 32768 tokens of 32 + 8 heads of 128 in bf16, 671 MB, take 123 us (5.4 TB/s); 25000 tokens of 20 prompts
// with 8 KV heads into pages, 206 MB, 33 us by the kernel trace (repeated passes, which may find data in the last-level cache), 40 a
// pass among others.  Small ones take 3.5 to 4.3 us, in which little more than loads that wait for each other (position, table
// entry, data) happens.
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

// A thread's two 16-byte pieces of a head: where they begin, their first planes and whether they turn.  The
// first pieces of a token's threads stand side by side, and so do the second ones, so that an access of a
// wavefront covers whole lines (two pieces side by side in each thread: 153 us for 32768 tokens where this
// takes 126, and 205 with the stores below).
struct Pieces {
  int lo, hi;         // elements
  int plane[2];       // adjacent planes: each piece holds its own; half layout: the same ones, half of them in each
  bool turn[2];
};
template <int N, int D, bool INTER>
__device__ __forceinline__ Pieces pieces(int c, int rot) {
  Pieces p;
  const int turning = INTER ? 0 : rot / (2 * N);  // threads that hold both halves of N planes
  if (c < turning) {
    p.lo = c * N;
    p.hi = rot / 2 + c * N;
    p.plane[0] = p.plane[1] = c * N;
    p.turn[0] = p.turn[1] = true;
  } else {
    const int first = INTER ? 0 : rot;
    p.lo = first + (c - turning) * N;
    p.hi = p.lo + (D - first) / 2;
    p.plane[0] = p.lo / 2;
    p.plane[1] = p.hi / 2;
    p.turn[0] = INTER && p.lo < rot;
    p.turn[1] = INTER && p.hi < rot;
  }
  return p;
}

// The factors of the thread's N planes at position pos (scale in both): N of the half layout, N / 2 of each piece
// of the other.
template <int N, bool INTER>
__device__ __forceinline__ void factors(const RopeView& r, const Pieces& p, int pos, bool grad, float (&cs)[N],
                                        float (&sn)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int h = INTER ? i / (N / 2) : 0;
    if (!p.turn[h]) continue;
    float co, si;
    turn_cos_sin(turn_rate(r.freq[p.plane[h] + (INTER ? i % (N / 2) : i)]), pos, co, si);
    cs[i] = co * r.scale;
    sn[i] = si * (grad ? -r.scale : r.scale);
  }
}

template <typename T, bool INTER>
__device__ __forceinline__ void turn(const Pieces& p, u32x4& lo, u32x4& hi, const float (&cs)[Vec<T>::N],
                                     const float (&sn)[Vec<T>::N]) {
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
  if (p.turn[0]) lo = Vec<T>::pack(x);
  if (p.turn[1]) hi = Vec<T>::pack(y);
}

// Stores that do not stay in the L2 (PAST): what is written here is read by a later launch.  They pay where a
// wavefront's store covers whole 64-byte runs (rope of 8192 tokens, 32 + 8 heads: 34.4 -> 27.1 us; 20 prompts of 25000 tokens
// to the cache: 45.8 -> 40.8) and cost where it does not (heads of 128 of which 32 turn, in halves: 46.4 -> 59.5).
template <bool PAST>
__device__ __forceinline__ void store(void* p, const u32x4& v) {
  if constexpr (PAST) __builtin_nontemporal_store(v, (u32x4*)p);
  else *(u32x4*)p = v;
}

template <typename T, int D, bool INTER, bool PAST>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a, FastDiv per_b, int hb) {
  constexpr int N = Vec<T>::N, TPT = D / (2 * N), TOK = kThreads / TPT;
  const int t = (int)blockIdx.x * TOK + (int)threadIdx.x / TPT;  // tokens of all batch entries in a row
  const int c = threadIdx.x % TPT;
  if (t >= a.batch * a.seq_len) return;
  const int b = fast_quot(per_b, t), s = t - b * a.seq_len;
  const Pieces p = pieces<N, D, INTER>(c, a.rope.rot);
  float cs[N], sn[N];
  const bool turns = p.turn[0] || p.turn[1];
  if (turns) {
    const int pos = a.positions ? a.positions[b * a.pos_stride + s] : a.start + s;
    factors<N, INTER>(a.rope, p, pos, a.grad, cs, sn);
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
      if (turns) turn<T, INTER>(p, lo[i], hi[i], cs, sn);
      store<PAST>(dst + p.lo, lo[i]);
      store<PAST>(dst + p.hi, hi[i]);
    }
  }
}

// A thread's planes of one token of every head of its share: K rotated, V copied.
template <typename T, int D, bool INTER, bool PAST>
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
  const Pieces p = pieces<N, D, INTER>(c, a.rope.rot);
  float cs[N], sn[N];
  const bool turns = p.turn[0] || p.turn[1];
  if (turns) factors<N, INTER>(a.rope, p, pos, false, cs, sn);
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
      if (turns) turn<T, INTER>(p, klo[j], khi[j], cs, sn);
      store<PAST>(kc + (h + j) * a.kc.sh + p.lo, klo[j]);
      store<PAST>(kc + (h + j) * a.kc.sh + p.hi, khi[j]);
      store<PAST>(vc + (h + j) * a.vc.sh + p.lo, vlo[j]);
      store<PAST>(vc + (h + j) * a.vc.sh + p.hi, vhi[j]);
    }
  }
}

// Heads per workgroup: at most `most`, fewer where that leaves the launch less than 2048 workgroups.
int head_share(int64_t tiles, int heads, int most) {
  int hb = most;
  while (hb > 1 && tiles * ((heads + hb - 1) / hb) < 2048) hb /= 2;
  return hb;
}

template <typename T, int D>
hipError_t rotate(const RotateArgs& a, hipStream_t s) {
  constexpr int TOK = kThreads / (D / (2 * Vec<T>::N));
  const int64_t tiles = ((int64_t)a.batch * a.seq_len + TOK - 1) / TOK;
  const int heads = a.heads_q + a.heads_kv;
  // (a workgroup of 32 tokens reads a run of each head, or, token-major, heads side by side: 32768 tokens of 32 + 8 heads
  // with 8 and 16 heads a workgroup take 126 and 132 us head-major, 158 and 138 token-major)
  const int hb = head_share(tiles, heads, a.q.sh < a.q.ss ? 16 : 8);
  const dim3 grid((unsigned)tiles, (unsigned)((heads + hb - 1) / hb));
  const FastDiv per_b = fast_div(a.seq_len);
  if (a.rope.interleaved) rotate_kernel<T, D, true, true><<<grid, kThreads, 0, s>>>(a, per_b, hb);
  else if (a.rope.rot * (int)sizeof(T) % 128 == 0) rotate_kernel<T, D, false, true><<<grid, kThreads, 0, s>>>(a, per_b, hb);
  else rotate_kernel<T, D, false, false><<<grid, kThreads, 0, s>>>(a, per_b, hb);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  constexpr int TOK = kThreads / (D / (2 * Vec<T>::N));
  const int64_t tiles = ((int64_t)a.batch * a.tokens + TOK - 1) / TOK;
  const int hb = head_share(tiles, a.heads_kv, 8);
  const dim3 grid((unsigned)tiles, (unsigned)((a.heads_kv + hb - 1) / hb));
  const FastDiv per_b = fast_div(a.tokens);
  if (a.rope.interleaved) append_kernel<T, D, true, true><<<grid, kThreads, 0, s>>>(a, per_b, hb);
  else if (a.rope.rot * (int)sizeof(T) % 128 == 0) append_kernel<T, D, false, true><<<grid, kThreads, 0, s>>>(a, per_b, hb);
  else append_kernel<T, D, false, false><<<grid, kThreads, 0, s>>>(a, per_b, hb);
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
