// paged_attn_kernels.hip -- attention of new tokens over a paged key-value cache.
//
// A new token's row of every query head of a KV group meets the same keys, so the
// G = heads_q / heads_kv heads (times the tokens, where a few drafted ones come
// together) are the columns of one matrix product with the cache: S^T = K Q^T,
// O^T = V^T P^T.  That is at most 2 * 32 operations a cached element, far below
// what the matrix cores do in the time HBM takes to bring it: the kernel is bound by
// reading K and V once, and everything else is arranged around that.
//
// Work.  The keys of every (sequence, KV head) are cut into units; all units of the
// call, in (sequence, head, key) order, are dealt out evenly to the workgroups, each
// taking one contiguous run.  Lengths are read on the device: unequal sequences
// balance themselves, and a captured launch stays right as they grow.  A run
// covers whole rows (their results are written at once) and at most one row's end
// and one row's beginning, which go to the workspace as partial results (O, running
// maximum, sum) and are joined in a fixed order by a second launch.
//
// A wavefront takes KT keys at a time (32 in bf16, 16 in fp32), its lanes holding K
// rows as the operand of S^T with no LDS in between: lane l reads 16-byte
// pieces of key row l % 16.  V arrives row-wise, 16 lanes to a row, and is the operand of
// O^T after an 8 x 8 transposition of 16-bit values in registers (bf16; fp32 operands hold one
// value, and need none).  The keys' order within a tile is chosen so that a lane's
// scores S^T are the very ones that its operand P^T of the second product needs.
//
// Precision: fp32 statistics and sums.  In bf16, P enters the second product in two
// bf16 parts, and so does a q that is rotated here: the matrix cores are idle most of
// the time, and o is then rounded once.
#include <algorithm>

#include "decode.h"

namespace seer {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kWorkers = 768;   // workgroups at most: three for each CU
constexpr int kMinUnits = 2;    // units a workgroup has at least, where there are several
constexpr int kWholeKeys = 512; // caches of at most this many tokens a sequence are never split
constexpr float kLn2 = 0.6931471805599453f;

struct KernelArgs {
  PagedArgs a;
  int group, rows, row_blocks;  // G, G tokens, blocks of 16 NT rows
  int capacity;                 // tokens that a table row has room for
  int unit;                     // keys per unit
  bool join;                    // rows may be split: records are written for the second launch
  float scale_log2;
  int2* record;                 // [batch heads_kv row_blocks] first slot and last workgroup of a split row, or -1
  float2* part_ml;              // [2 kWorkers][16 NT] maximum and sum
  float* part_o;                // [2 kWorkers][16 NT][D]
};

template <typename T, int D>
struct Shape;
template <int D>
struct Shape<uint16_t, D> {
  static constexpr int KT = 32;       // keys of a tile
  static constexpr int KSUB = 2;      // K row groups of 16
  static constexpr int KCH = D / 32;  // 16-byte pieces of a K row per lane
  static constexpr int PK = 8;        // keys of a lane in S^T, P^T and V
  static constexpr int VW = D / 32;   // dwords of a V row per lane
  static constexpr int VP = 1;        // pieces they come in
};
template <int D>
struct Shape<float, D> {
  static constexpr int KT = 16, KSUB = 1, KCH = D / 16, PK = 4, VW = D / 16, VP = D / 64;
};

// Keys that the tokens of a sequence see at most.
__device__ __forceinline__ int length_of(const KernelArgs& k, int b) {
  int len = 0;
  const int32_t* p = k.a.positions + b * k.a.pos_stride;
  for (int s = 0; s < k.a.tokens; ++s) len = max(len, min(p[s], k.capacity - 1) + 1);
  return len;
}
__device__ __forceinline__ int units_of(const KernelArgs& k, int b) {
  return max(1, (int)(((int64_t)length_of(k, b) + k.unit - 1) / k.unit));
}

// The units dealt to the workgroups: workgroup w has base (+ 1 for the first `rest`).
struct Deal {
  int64_t base, rest;
  int workers;
  __device__ __forceinline__ int64_t first(int w) const { return w * base + min((int64_t)w, rest); }
  __device__ __forceinline__ int owner(int64_t x) const {
    const int64_t big = rest * (base + 1);
    return (int)(x < big ? x / (base + 1) : rest + (x - big) / base);
  }
};

// A tile's operands as a lane holds them.
template <typename T, int D>
struct Tile {
  using S = Shape<T, D>;
  u32x4 k[S::KSUB][S::KCH];
  uint32_t v[S::PK][S::VW];
  uint32_t there;  // bit e: key e of the lane's PK is seen and its page exists
};

template <typename T, int D, int NT, int QP, bool OCT>
__global__ __launch_bounds__(kThreads) void paged_attn_kernel(KernelArgs ka) {
  using S = Shape<T, D>;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NA = D / 16;          // accumulators of a column tile
  constexpr int ROWS = 16 * NT;
  constexpr int OSTR = D + 4;
  __shared__ __attribute__((aligned(16))) float sO[kWaves][ROWS][OSTR];
  __shared__ float sM[kWaves][ROWS], sL[kWaves][ROWS];
  __shared__ int sScan[kWaves];
  __shared__ int sB;
  __shared__ int64_t sOff;

  const PagedArgs& a = ka.a;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane % 16, g = lane / 16;
  const int items = a.heads_kv * ka.row_blocks;  // rows of a sequence
  const float c = ka.scale_log2;

  // ---- this workgroup's run of units
  const int share = (a.batch + kThreads - 1) / kThreads;  // sequences per thread
  const int b_lo = min(tid * share, a.batch), b_hi = min(b_lo + share, a.batch);
  int mine = 0;
  for (int b = b_lo; b < b_hi; ++b) mine += units_of(ka, b);
  int upto = mine;  // inclusive prefix over the threads
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int y = __shfl_up(upto, off);
    if (lane >= off) upto += y;
  }
  if (lane == kWave - 1) sScan[wave] = upto;
  __syncthreads();
  int all = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) upto += sScan[w];
    all += sScan[w];
  }
  const int64_t total = (int64_t)all * items;
  Deal deal;
  deal.workers = (int)max((int64_t)1, min((int64_t)gridDim.x, total / kMinUnits));
  if (!ka.join) deal.workers = (int)min((int64_t)gridDim.x, total);
  const int w = blockIdx.x;
  if (w >= deal.workers) return;
  deal.base = total / deal.workers;
  deal.rest = total - deal.base * deal.workers;
  int64_t x = deal.first(w);
  const int64_t x_end = deal.first(w + 1);
  {
    int64_t before = (int64_t)(upto - mine) * items;
    if (x >= before && x < (int64_t)upto * items) {
      int b = b_lo;
      for (; b < b_hi - 1; ++b) {
        const int64_t next = before + (int64_t)units_of(ka, b) * items;
        if (x < next) break;
        before = next;
      }
      sB = b;
      sOff = x - before;
    }
  }
  __syncthreads();
  int b = sB;
  int row_units = units_of(ka, b);
  int item = (int)(sOff / row_units);
  int u0 = (int)(sOff - (int64_t)item * row_units);
  bool first_run = true;

  for (; x < x_end;) {
    const int take = (int)min((int64_t)(row_units - u0), x_end - x);
    const int h = item / ka.row_blocks, rb = item - h * ka.row_blocks;
    const int r0 = rb * ROWS;                      // the first row of the block
    const int nrows = min(ROWS, ka.rows - r0);
    const bool whole = take == row_units;
    const int32_t* pos_b = a.positions + b * a.pos_stride;

    // ---- the columns: rows r0 + 16 ct + n, the last key each sees
    int last[NT], token[NT];
    int most = -1, least = 0x7fffffff;
    const T* qp[NT];
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) {
      const int r = min(r0 + 16 * ct + n, ka.rows - 1);
      const int t = r / ka.group;
      token[ct] = t;
      const int p = min(pos_b[t], ka.capacity - 1);
      last[ct] = p;
      most = max(most, p);
      if (p >= 0) least = min(least, p);
      qp[ct] = (const T*)a.q.ptr + b * a.q.sb + (h * ka.group + (r - t * ka.group)) * a.q.sh + t * a.q.ss;
    }
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) {
      most = max(most, __shfl_xor(most, off));
      least = min(least, __shfl_xor(least, off));
    }
    const int len = __builtin_amdgcn_readfirstlane(most + 1);
    const int common = __builtin_amdgcn_readfirstlane(most < 0 ? 0 : least + 1);  // keys that every live row sees
    const int64_t k_lo = (int64_t)u0 * ka.unit;
    const int k_hi = (int)min((int64_t)len, k_lo + (int64_t)take * ka.unit);
    // tiles below `even` are seen alike by all live rows
    const int even = common == len ? k_hi : min(k_hi, common / S::KT * S::KT);

    // ---- Q^T operand, in QP parts
    constexpr int QJ = BF ? D / 32 : D / 16;
    u32x4 q[QP][NT][QJ];
    if (a.rope.freq != nullptr) {
      // a thread rotates 8 elements of one row, then the operands are read back
      for (int e = tid; e < ROWS * (D / 8); e += kThreads) {
        const int rl = e / (D / 8), d0 = e % (D / 8) * 8;
        const int r = min(r0 + rl, ka.rows - 1), t = r / ka.group;
        const T* src = (const T*)a.q.ptr + b * a.q.sb + (h * ka.group + (r - t * ka.group)) * a.q.sh + t * a.q.ss;
        const int half = a.rope.rot / 2;
        const int pos = pos_b[t];
        const bool turns = d0 < a.rope.rot, second = d0 >= half;
        float own[8], other[8];
        auto load8 = [&](int d, float(&y)[8]) {
          if constexpr (BF) {
            const u32x4 z = *(const u32x4*)(src + d);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              y[2 * i] = __uint_as_float(z[i] << 16);
              y[2 * i + 1] = __uint_as_float(z[i] & 0xffff0000u);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = src[d + i];
          }
        };
        load8(d0, own);
        if (turns) {
          if (a.rope.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float co, si;
              turn_cos_sin(turn_rate(a.rope.freq[d0 / 2 + i]), pos, co, si);
              co *= a.rope.scale;
              si *= a.rope.scale;
              const float u = own[2 * i], v = own[2 * i + 1];
              own[2 * i] = u * co - v * si;
              own[2 * i + 1] = u * si + v * co;
            }
          } else {
            load8(second ? d0 - half : d0 + half, other);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float co, si;
              turn_cos_sin(turn_rate(a.rope.freq[(second ? d0 - half : d0) + i]), pos, co, si);
              own[i] = own[i] * (co * a.rope.scale) + other[i] * ((second ? si : -si) * a.rope.scale);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sO[0][rl][d0 + i] = own[i];
      }
      __syncthreads();
#pragma unroll
      for (int ct = 0; ct < NT; ++ct)
#pragma unroll
        for (int j = 0; j < QJ; ++j) {
          if constexpr (BF) {
            const float* z = &sO[0][16 * ct + n][32 * j + 8 * g];
            union {
              bf16x8 v;
              u32x4 r;
            } hi, lo;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              hi.v[i] = (__bf16)z[i];
              lo.v[i] = (__bf16)(z[i] - (float)hi.v[i]);
            }
            q[0][ct][j] = hi.r;
            if constexpr (QP == 2) q[1][ct][j] = lo.r;
          } else {
            q[0][ct][j] = *(const u32x4*)&sO[0][16 * ct + n][16 * j + 4 * g];
          }
        }
      __syncthreads();  // sO is free again
    } else {
#pragma unroll
      for (int ct = 0; ct < NT; ++ct)
#pragma unroll
        for (int j = 0; j < QJ; ++j)
          q[0][ct][j] = *(const u32x4*)(qp[ct] + (BF ? 32 * j + 8 * g : 16 * j + 4 * g));
    }

    f32x4 acc[NT][NA];
#pragma unroll
    for (int ct = 0; ct < NT; ++ct)
#pragma unroll
      for (int i = 0; i < NA; ++i) acc[ct][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m[NT], l[NT];
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) m[ct] = -INFINITY, l[ct] = 0.f;

    const T* kbase = (const T*)a.kc.ptr + h * a.kc.sh;
    const T* vbase = (const T*)a.vc.ptr + h * a.vc.sh;
    const int32_t* table = a.table.ptr + b * a.table.stride;

    // page and slot of a key; false (page 0, slot 0) where there is none
    auto find = [&](int key, int64_t& page, int64_t& slot) -> bool {
      const int i = fast_quot(a.table.page, key);
      const int p = key < len ? table[i] : -1;
      const bool ok = p >= 0 && p < a.table.num_pages;
      page = ok ? p : 0;
      slot = ok ? key - i * a.table.page.d : 0;
      return ok;
    };

    using TileT = Tile<T, D>;
    auto load = [&](TileT& t, int key0) {
      // K: lane row r = n of sub-tile i is key 8 (r / 4) + 4 i + r % 4 (bf16), r (fp32)
      const int kk = BF ? n / 4 * 8 + n % 4 : n;
      const T* kp[S::KSUB];
      if constexpr (OCT) {  // pages hold whole aligned runs of 8 keys: one look-up for each run
        int64_t page, slot;
        find(key0 + kk / 8 * 8, page, slot);
#pragma unroll
        for (int i = 0; i < S::KSUB; ++i) kp[i] = kbase + page * a.kc.sp + (slot + kk % 8 + 4 * i) * a.kc.ss;
      } else {
#pragma unroll
        for (int i = 0; i < S::KSUB; ++i) {
          int64_t page, slot;
          find(key0 + kk + 4 * i, page, slot);
          kp[i] = kbase + page * a.kc.sp + slot * a.kc.ss;
        }
      }
#pragma unroll
      for (int i = 0; i < S::KSUB; ++i)
#pragma unroll
        for (int j = 0; j < S::KCH; ++j) t.k[i][j] = *(const u32x4*)(kp[i] + (BF ? 32 * j + 8 * g : 16 * j + 4 * g));
      // V: the lane's keys are PK g + e
      const int vk = S::PK * g;
      t.there = 0;
      const T* vp = vbase;
      if constexpr (OCT) {
        int64_t page, slot;
        const bool ok = find(key0 + vk / 8 * 8, page, slot);
        vp = vbase + page * a.vc.sp + (slot + vk % 8) * a.vc.ss;
        if (ok) {
          const int seen = min(max(len - (key0 + vk), 0), S::PK);
          t.there = (1u << seen) - 1u;
        }
      }
#pragma unroll
      for (int e = 0; e < S::PK; ++e) {
        const T* p = vp + e * a.vc.ss;
        if constexpr (!OCT) {
          int64_t page, slot;
          if (find(key0 + vk + e, page, slot)) t.there |= 1u << e;
          p = vbase + page * a.vc.sp + slot * a.vc.ss;
        }
        if constexpr (BF && S::VW == 4) {
          const u32x4 z = *(const u32x4*)(p + 8 * n);
#pragma unroll
          for (int i = 0; i < 4; ++i) t.v[e][i] = z[i];
        } else if constexpr (BF) {
          const u32x2 z = *(const u32x2*)(p + 4 * n);
          t.v[e][0] = z[0];
          t.v[e][1] = z[1];
        } else {
#pragma unroll
          for (int f = 0; f < S::VP; ++f) {
            const u32x4 z = *(const u32x4*)(p + 64 * f + 4 * n);
#pragma unroll
            for (int i = 0; i < 4; ++i) t.v[e][4 * f + i] = z[i];
          }
        }
      }
    };

    // S^T of a column tile: element e is key key0 + PK g + e of the lane's column
    auto scores = [&](const TileT& t, int ct, float (&s)[S::PK]) {
#pragma unroll
      for (int i = 0; i < S::KSUB; ++i) {
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int part = QP - 1; part >= 0; --part)
#pragma unroll
          for (int j = 0; j < S::KCH; ++j) {
            if constexpr (BF) {
              y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[i][j]),
                                                          __builtin_bit_cast(bf16x8, q[part][ct][j]), y, 0, 0, 0);
            } else {
#pragma unroll
              for (int f = 0; f < 4; ++f)
                y = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.k[i][j][f]),
                                                         __uint_as_float(q[part][ct][j][f]), y, 0, 0, 0);
            }
          }
#pragma unroll
        for (int f = 0; f < 4; ++f) s[4 * i + f] = y[f];
      }
    };

    // running maximum and sum; s becomes P
    auto softmax = [&](int ct, float (&s)[S::PK]) {
      float mx = s[0];
#pragma unroll
      for (int e = 1; e < S::PK; ++e) mx = fmaxf(mx, s[e]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (__ballot(mx > m[ct]) != 0) {
        const float m_new = fmaxf(m[ct], mx);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[ct] - m_new) * c);
        m[ct] = m_new;
        l[ct] *= alpha;
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int f = 0; f < 4; ++f) acc[ct][i][f] *= alpha;
      }
      // (the difference first: the largest score's weight is 1 exactly, however large it is)
      const float m0 = m[ct] == -INFINITY ? 0.f : m[ct];
#pragma unroll
      for (int e = 0; e < S::PK; ++e) {
        s[e] = __builtin_amdgcn_exp2f((s[e] - m0) * c);
        l[ct] += s[e];
      }
    };

    // o += V^T P^T; accumulator i, element f of the lane: column n, feature
    // (4 g + f) D/16 + i (bf16), 64 (i / 4) + 4 (4 g + f) + i % 4 (fp32)
    auto product = [&](const TileT& t, const float (&p)[S::PK], f32x4 (&o)[NA]) {
      if constexpr (BF) {
        bf16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          hi[e] = (__bf16)p[e];
          lo[e] = (__bf16)(p[e] - (float)hi[e]);
        }
#pragma unroll
        for (int i = 0; i < NA; ++i) {
          u32x4 z;
#pragma unroll
          for (int f = 0; f < 4; ++f)
            z[f] = __builtin_amdgcn_perm(t.v[2 * f + 1][i / 2], t.v[2 * f][i / 2], i % 2 ? 0x07060302u : 0x05040100u);
          const bf16x8 vt = __builtin_bit_cast(bf16x8, z);
          o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, lo, o[i], 0, 0, 0);
          o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, hi, o[i], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int e = 0; e < S::PK; ++e)
#pragma unroll
          for (int i = 0; i < NA; ++i)
            o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[e][i]), p[e], o[i], 0, 0, 0);
      }
    };

    constexpr int STEP = kWaves * S::KT;
    int key0 = (int)k_lo + wave * S::KT;
    for (; key0 < even; key0 += STEP) {
      TileT t;
      load(t, key0);
      const bool full = __ballot(t.there != (1u << S::PK) - 1u) == 0;
      if (!full) {  // what stands in slots that no row sees may be anything
#pragma unroll
        for (int e = 0; e < S::PK; ++e)
          if (!(t.there >> e & 1))
#pragma unroll
            for (int i = 0; i < S::VW; ++i) t.v[e][i] = 0;
      }
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) {
        float s[S::PK];
        scores(t, ct, s);
        if (!full)
#pragma unroll
          for (int e = 0; e < S::PK; ++e) s[e] = t.there >> e & 1 ? s[e] : -INFINITY;
        softmax(ct, s);
        product(t, s, acc[ct]);
      }
    }
    // the keys near the new tokens, where the tokens' rows see different ones: a key that
    // one token does not see must not reach its output even as 0 times whatever V holds
    for (; key0 < k_hi; key0 += STEP) {
      TileT t;
      load(t, key0);
      const int lane_key = key0 + S::PK * g;
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) {
        float s[S::PK];
        scores(t, ct, s);
#pragma unroll
        for (int e = 0; e < S::PK; ++e)
          s[e] = (t.there >> e & 1) && lane_key + e <= last[ct] ? s[e] : -INFINITY;
        softmax(ct, s);
        const int t_lo = min(r0 + 16 * ct, ka.rows - 1) / ka.group, t_hi = min(r0 + 16 * ct + 15, ka.rows - 1) / ka.group;
        for (int tk = t_lo; tk <= t_hi; ++tk) {
          const int lk = min(pos_b[tk], ka.capacity - 1);
          TileT seen;
#pragma unroll
          for (int e = 0; e < S::PK; ++e)
#pragma unroll
            for (int i = 0; i < S::VW; ++i) seen.v[e][i] = (t.there >> e & 1) && lane_key + e <= lk ? t.v[e][i] : 0;
          f32x4 o[NA];
#pragma unroll
          for (int i = 0; i < NA; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
          product(seen, s, o);
          if (token[ct] == tk)
#pragma unroll
            for (int i = 0; i < NA; ++i) acc[ct][i] += o[i];
        }
      }
    }

    // ---- the wavefronts' results together
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) {
      l[ct] += __shfl_xor(l[ct], 16);
      l[ct] += __shfl_xor(l[ct], 32);
      const int col = 16 * ct + n;
      if (g == 0) {
        sM[wave][col] = m[ct];
        sL[wave][col] = l[ct];
      }
#pragma unroll
      for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const int d = BF ? (4 * g + f) * NA + i : 64 * (i / 4) + 4 * (4 * g + f) + i % 4;
          sO[wave][col][d] = acc[ct][i][f];
        }
    }
    __syncthreads();
    const int slot = 2 * w + (first_run ? 0 : 1);
    for (int e = tid; e < nrows * (D / 4); e += kThreads) {
      const int rl = e / (D / 4), d = e % (D / 4) * 4;
      float mx = sM[0][rl];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) mx = fmaxf(mx, sM[i][rl]);
      float sum = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float wgt = sM[i][rl] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((sM[i][rl] - mx) * c);
        sum += wgt * sL[i][rl];
        o += wgt * *(const f32x4*)&sO[i][rl][d];
      }
      if (!whole) {
        *(f32x4*)(ka.part_o + ((int64_t)slot * ROWS + rl) * D + d) = o;
        if (d == 0) ka.part_ml[(int64_t)slot * ROWS + rl] = make_float2(mx, sum);
        continue;
      }
      const int r = r0 + rl, t = r / ka.group, hq = h * ka.group + (r - t * ka.group);
      const bool none = sum == 0.f || pos_b[t] < 0;
      const float inv = none ? 0.f : 1.f / sum;
      T* out = (T*)a.o + b * a.osb + hq * a.osh + t * a.oss + d;
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const float y = none ? 0.f : o[f] * inv;
        if constexpr (BF) ((__bf16*)out)[f] = (__bf16)y;
        else out[f] = y;
      }
      if (a.lse != nullptr && d == 0)
        a.lse[((int64_t)b * a.heads_q + hq) * a.tokens + t] =
            none ? -INFINITY : ((mx == -INFINITY ? 0.f : mx * c) + __log2f(sum)) * kLn2;
    }
    if (ka.join && u0 == 0 && tid == 0)
      ka.record[(int64_t)b * items + item] =
          whole ? make_int2(-1, -1) : make_int2(slot, deal.owner(x + row_units - 1));
    __syncthreads();

    first_run = false;
    x += take;
    u0 += take;
    if (u0 == row_units) {
      u0 = 0;
      if (++item == items) {
        item = 0;
        ++b;
        if (x < x_end) row_units = units_of(ka, b);
      }
    }
  }
}

// One row (a token of a query head) whose keys several workgroups shared: their partial
// results, in the order of the keys.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(KernelArgs ka, int rows_block) {
  constexpr int V4 = D / 4, GRP = kThreads / V4;
  __shared__ float sW[kWorkers];
  __shared__ float sR[kWaves], sS[kWaves];
  __shared__ __attribute__((aligned(16))) float sO[GRP][D];
  const PagedArgs& a = ka.a;
  const int64_t at = blockIdx.x;
  const int2 rec = ka.record[at];
  if (rec.x < 0) return;
  const int items = a.heads_kv * ka.row_blocks;
  const int b = (int)(at / items), item = (int)(at - (int64_t)b * items);
  const int h = item / ka.row_blocks, rb = item - h * ka.row_blocks;
  const int rl = blockIdx.y, r = rb * rows_block + rl;
  if (r >= ka.rows) return;
  const int w0 = rec.x / 2, parts = rec.y - w0 + 1;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  auto slot = [&](int p) { return (int64_t)(p == 0 ? rec.x : 2 * (w0 + p)) * rows_block + rl; };
  const float c = ka.scale_log2;

  float mx = -INFINITY;
  for (int p = tid; p < parts; p += kThreads) mx = fmaxf(mx, ka.part_ml[slot(p)].x);
  mx = wave_max(mx);
  if (lane == 0) sR[wave] = mx;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) mx = fmaxf(mx, sR[i]);
  float sum = 0.f;
  for (int p = tid; p < parts; p += kThreads) {
    const float2 ml = ka.part_ml[slot(p)];
    const float wgt = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml.x - mx) * c);
    sW[p] = wgt;
    sum += wgt * ml.y;
  }
  sum = wave_sum(sum);
  if (lane == 0) sS[wave] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) sum += sS[i];

  const int d = tid % V4 * 4, grp = tid / V4;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int p = grp; p < parts; p += GRP) o += sW[p] * *(const f32x4*)(ka.part_o + slot(p) * D + d);
  *(f32x4*)&sO[grp][d] = o;
  __syncthreads();
  const int t = r / ka.group, hq = h * ka.group + (r - t * ka.group);
  const bool none = sum == 0.f || a.positions[b * a.pos_stride + t] < 0;
  if (tid < D) {
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < GRP; ++i) y += sO[i][tid];
    y = none ? 0.f : y / sum;
    T* out = (T*)a.o + b * a.osb + hq * a.osh + t * a.oss + tid;
    if constexpr (sizeof(T) == 2) *(__bf16*)out = (__bf16)y;
    else *out = y;
  }
  if (a.lse != nullptr && tid == 0)
    a.lse[((int64_t)b * a.heads_q + hq) * a.tokens + t] =
        none ? -INFINITY : ((mx == -INFINITY ? 0.f : mx * c) + __log2f(sum)) * kLn2;
}

struct Plan {
  int group, rows, nt, row_blocks;
  size_t ml, o, total;  // byte offsets in the workspace (the records come first)
};
Plan plan(int batch, int heads_q, int heads_kv, int tokens, int head_dim) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  Plan p;
  p.group = heads_q / heads_kv;
  p.rows = p.group * tokens;
  p.nt = p.rows > 16 ? 2 : 1;
  p.row_blocks = (p.rows + 16 * p.nt - 1) / (16 * p.nt);
  p.ml = up((size_t)batch * heads_kv * p.row_blocks * sizeof(int2));
  p.o = p.ml + up((size_t)2 * kWorkers * 16 * p.nt * sizeof(float2));
  p.total = p.o + (size_t)2 * kWorkers * 16 * p.nt * head_dim * sizeof(float);
  return p;
}

template <typename T, int D, int NT, int QP>
hipError_t launch(const KernelArgs& k, dim3 grid, hipStream_t s) {
  if (k.a.table.page.d % 8 == 0) paged_attn_kernel<T, D, NT, QP, true><<<grid, kThreads, 0, s>>>(k);
  else paged_attn_kernel<T, D, NT, QP, false><<<grid, kThreads, 0, s>>>(k);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_typed(const KernelArgs& k, int nt, dim3 grid, hipStream_t s) {
  hipError_t e;
  if constexpr (sizeof(T) == 2) {
    if (k.a.rope.freq) e = nt == 2 ? launch<T, D, 2, 2>(k, grid, s) : launch<T, D, 1, 2>(k, grid, s);
    else e = nt == 2 ? launch<T, D, 2, 1>(k, grid, s) : launch<T, D, 1, 1>(k, grid, s);
  } else {
    e = nt == 2 ? launch<T, D, 2, 1>(k, grid, s) : launch<T, D, 1, 1>(k, grid, s);
  }
  if (e != hipSuccess || !k.join) return e;
  const int64_t rows = (int64_t)k.a.batch * k.a.heads_kv * k.row_blocks;
  paged_join_kernel<T, D><<<dim3((unsigned)rows, (unsigned)std::min(k.rows, 16 * nt)), kThreads, 0, s>>>(k, 16 * nt);
  return hipGetLastError();
}

}  // namespace

size_t paged_attn_workspace(int batch, int heads_q, int heads_kv, int tokens, int head_dim) {
  return plan(batch, heads_q, heads_kv, tokens, head_dim).total;
}

hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t s) {
  const Plan p = plan(a.batch, a.heads_q, a.heads_kv, a.tokens, a.head_dim);
  KernelArgs k;
  k.a = a;
  k.group = p.group;
  k.rows = p.rows;
  k.row_blocks = p.row_blocks;
  k.capacity = a.table.max_pages * a.table.page.d;  // (at most 2^30: no sum of keys overflows)
  const int step = kWaves * (a.bf16 ? 32 : 16);
  const int64_t items = (int64_t)a.heads_kv * p.row_blocks;
  int64_t unit = step;
  k.join = k.capacity > kWholeKeys;
  if (!k.join) unit = (k.capacity + step - 1) / step * step;
  // (counts of units stay below 2^31)
  auto units = [&]() { return (k.capacity + unit - 1) / unit; };
  while (units() * std::max((int64_t)a.batch, items) > INT32_MAX / 2 && unit < (1 << 29)) unit *= 2;
  k.unit = (int)unit;
  k.scale_log2 = a.scale * kLog2e;
  char* ws = (char*)a.workspace;
  k.record = (int2*)ws;
  k.part_ml = (float2*)(ws + p.ml);
  k.part_o = (float*)(ws + p.o);
  const dim3 grid((unsigned)std::min((int64_t)kWorkers, units() * items * a.batch));
  if (a.bf16) return a.head_dim == 128 ? launch_typed<uint16_t, 128>(k, p.nt, grid, s) : launch_typed<uint16_t, 64>(k, p.nt, grid, s);
  return a.head_dim == 128 ? launch_typed<float, 128>(k, p.nt, grid, s) : launch_typed<float, 64>(k, p.nt, grid, s);
}

}  // namespace seer
