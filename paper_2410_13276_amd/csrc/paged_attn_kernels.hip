// paged_attn_kernels.hip -- attention of new tokens over a paged key-value cache.
//
// A new token's row of every query head of a KV group meets the same keys, so the
// G = heads_q / heads_kv heads (times the tokens, where a few drafted ones come
// together) are the columns of one matrix product with the cache: S^T = K Q^T,
// O^T = V^T P^T.  That is at most 2 * 32 operations a cached element, far below
// what the matrix cores do in the time HBM takes to bring it (they are busy 11% of the time with 4
// columns): the kernel is bound by reading K and V once, and everything else is arranged around
// that.  A token after 131072 tokens (32 / 8 heads of 128, bf16) reads 537 MB in 93 us, 64 sequences of 200 to 16000
// tokens 955 MB in 169 us (5.8 and 5.7 TB/s; a kernel that only reads takes 87 and 159 us, a copy moves 5.1 TB/s).
// Without any of the arithmetic the first takes 1% less.
//
// Work.  The keys of every (sequence, KV head) are cut into units of a tile for each
// wavefront; all units of the call, in (sequence, head, key) order, are dealt out evenly to the
// workgroups, each taking one contiguous run.  Lengths are read on the device: unequal sequences
// balance themselves, and a captured launch stays right as they grow.  A run
// covers whole rows (their results are written at once) and at most one row's end
// and one row's beginning, which go to the workspace as partial results (O, running
// maximum, sum) and are joined in a fixed order by a second launch (no counter to set up, and the
// same bits every time).
//
// A wavefront takes KT keys at a time (32 in bf16, 16 in fp32), its lanes holding K
// rows as the operand of S^T with no LDS in between: lane l reads 16-byte
// pieces of key row l % 16.  V arrives row-wise, 16 lanes to a row, and is the operand of
// O^T after an 8 x 8 transposition of 16-bit values in registers (bf16; fp32 operands hold one
// value, and need none).  The keys' order within a tile is chosen so that a lane's
// scores S^T are the very ones that its operand P^T of the second product needs.  Only Q^T is read
// from the LDS, a tile at a time: the registers hold the tile, the accumulators and loads in flight.
//
// Precision: fp32 statistics and sums.  In bf16, P enters the second product in three bf16 parts, which hold fp32 whole, and
// so does a q that is rotated here the first; o is then rounded once.  The matrix cores are idle most of the time: two parts
// of q cost 0.3 us less for a token after 2000 tokens and 1.2 of 58 for four drafted ones, and left the log-sum-exp up to
// 1.2e-5 off where this leaves 1.5e-6; two of P cost 0.2 us and 1.3 of 51 less, and gave 0.08 to 0.2% of o's elements
// another last bit than the same formula wholly in fp32 does, where this gives at most 0.07%.
#include <algorithm>

#include "decode.h"

namespace seer {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kWorkers = 512;   // workgroups at most: two for each CU
// Rows are not split, and the second launch not made, where a row has room for so many keys at most (fp32: half), and
// for twice as many where 128 rows or more, but not more than workgroups, share the launch.  Whole against split, 32 / 8
// heads of 128: 1 sequence of 400 tokens 10.7 and 11.9 us, of 900 15.3 and 11.9; 16 of 900 17.1 and 19.3; 64 of 900 47.5 and
// 49.5; fp32, 8 / 8 heads of 64, 1 of 400 11.0 and 9.3, 64 of 400 20.9 and 22.7.
constexpr int kWholeKeys = 512;
constexpr float kLn2 = 0.6931471805599453f;

struct Stride16 {
  uint32_t page, slot;
};

struct KernelArgs {
  PagedArgs a;
  Stride16 kst, vst;            // strides of the pools, in 16-byte pieces
  int rows, row_blocks;         // G tokens, blocks of 16 NT rows
  FastDiv group, blocks;        // by G and row_blocks
  int capacity;                 // tokens that a table row has room for
  int unit_shift;               // log2 of the keys per unit
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
__device__ __forceinline__ int units_of(const KernelArgs& k, int len) {
  return max(1, (len + (1 << k.unit_shift) - 1) >> k.unit_shift);
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

// A tile's operands as a lane holds them.
template <typename T, int D>
struct Tile {
  using S = Shape<T, D>;
  u32x4 k[S::KSUB][S::KCH];
  uint32_t v[S::PK][S::VW];
  uint32_t there;  // bit e: key e of the lane's PK is seen and its page exists
};

template <typename T, int D, int NT, int QP, bool OCT>
__global__ __launch_bounds__(kThreads, 2) void paged_attn_kernel(KernelArgs ka) {
  using S = Shape<T, D>;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NA = D / 16;          // accumulators of a column tile
  constexpr int ROWS = 16 * NT;
  // A row's beginning and end, in units: what it weighs beside its units (64 sequences of 200 to 16000 tokens: 186 us
  // without, 177 with 1, 181 with 2; four drafted tokens on two column tiles: 55.0, 50.6, 50.4)
  constexpr int kRowCost = NT;
  constexpr int OSTR = D + 4;
  constexpr int QJ = BF ? D / 32 : D / 16;
  // Partial sums of an fp32 score, joined by pairs: one chain of D sums rounds off twice as far (o of 1000 keys on average
  // 5.2e-7 off, with two sums 3.1e-7, with four 2.6e-7).  Beside two column tiles of 128 features four of them spill (28 / 4
  // heads, four tokens: 94.7 us, with two sums 92.6, with one 92.9; 24 / 1 heads 41.8, 39.7 and 40.0).
  constexpr int SUMS = BF ? 1 : NT == 2 && D == 128 ? 2 : 4;
  // the operand Q^T as the lanes read it and the tokens' cosines and sines, then the wavefronts' results
  __shared__ union {
    struct {
      u32x4 q[QP][NT][QJ][kWave];
      float2 cs[ROWS][D / 2];
    };
    float o[kWaves][ROWS][OSTR];
  } sh;
  __shared__ float sM[kWaves][ROWS], sL[kWaves][ROWS];

  const PagedArgs& a = ka.a;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane % 16, g = lane / 16;
  const int items = a.heads_kv * ka.row_blocks;  // rows of a sequence
  const int group = ka.group.d;
  const float c = ka.scale_log2;

  // (every line of the arguments is fetched now, not when it is first needed)
  asm volatile("" ::"s"(a.osb), "s"(a.kc.ptr), "s"(a.table.ptr), "s"(a.batch), "s"(ka.kst.page), "s"(ka.part_o));

  const bool rope = QP == 3 || (!BF && a.rope.freq != nullptr);
  // angle per position of plane `lane` (no branch around the load: it would be waited for at once)
  const double freq = (rope ? a.rope.freq : (const double*)a.kc.ptr)[rope ? min(lane, a.rope.rot / 2 - 1) : 0];

  // ---- this workgroup's share.  Every wavefront works it out by itself: a lane sums the weights of some
  // sequences in a row, and a scan over the lanes finds the sequence that the share begins in.
  const int share = (a.batch + kWave - 1) / kWave;  // sequences per lane
  const int b_lo = min(lane * share, a.batch), b_hi = min(b_lo + share, a.batch);
  int mine = 0, my_len = 0;
  for (int i = b_lo; i < b_hi; ++i) {
    my_len = length_of(ka, i);
    mine += units_of(ka, my_len) + kRowCost;
  }
  const int upto = wave_prefix(mine);
  TurnRate rate = turn_rate(freq);
  asm volatile("" : "+v"(rate.hi), "+v"(rate.lo));  // (here: the positions' wait was its wait too; later it would be the tile's)
  const int w = blockIdx.x;
  const Deal deal((uint32_t)(__builtin_amdgcn_readlane(upto, kWave - 1) * items), gridDim.x);
  if (w >= (int)deal.workers) return;
  int x = deal.first(w);
  const int x_end = deal.first(w + 1);
  const int owner_lane = (int)__popcll(__ballot(upto * items <= x));
  int b = owner_lane * share;
  int off = x - (__builtin_amdgcn_readlane(upto, owner_lane) - __builtin_amdgcn_readlane(mine, owner_lane)) * items;
  int len = share == 1 ? __builtin_amdgcn_readlane(my_len, owner_lane) : length_of(ka, b);
  int row_units = units_of(ka, len);
  while (off >= (row_units + kRowCost) * items) {
    off -= (row_units + kRowCost) * items;
    len = length_of(ka, ++b);
    row_units = units_of(ka, len);
  }
  len = __builtin_amdgcn_readfirstlane(len);
  row_units = __builtin_amdgcn_readfirstlane(row_units);
  int item = (int)((uint32_t)off / (uint32_t)(row_units + kRowCost));
  int at_w = off - item * (row_units + kRowCost);  // position within the row's weight

  // ---- a run of one row's units [u0, u1): where it is, and its first tile
  int u0, u1, h, key0, k_hi;
  const char *kbase, *vbase;
  const int32_t* table;

  // The pages of a lane's keys of a tile, fetched a tile ahead of its loads.  K: lane row n
  // of sub-tile i is key 8 (n / 4) + 4 i + n % 4 (bf16), n (fp32); V: keys PK g + e.  Where pages hold
  // whole aligned runs of 8 keys (OCT) one look-up serves a run.
  const int kk = BF ? n / 4 * 8 + n % 4 : n;
  const int vk = S::PK * g;
  struct Pages {
    int k[OCT ? 1 : S::KSUB], v[OCT ? 1 : S::PK];
  };
  // (A key past the run is looked up at the run's last one and then has no page: no branch, and loads that are
  // not wanted all go to the pool's first slots.)
  auto page_of = [&](int key) -> int {
    const int page = table[fast_quot(a.table.page, max(min(key, k_hi - 1), 0))];
    return key < k_hi ? page : -1;
  };
  auto pages = [&](int key0) -> Pages {
    Pages p;
    if constexpr (OCT) {
      p.k[0] = page_of(key0 + kk / 8 * 8);  // (the run's first key: it exists where any of them does)
      p.v[0] = page_of(key0 + vk / 8 * 8);
    } else {
#pragma unroll
      for (int i = 0; i < S::KSUB; ++i) p.k[i] = page_of(key0 + kk + 4 * i);
#pragma unroll
      for (int e = 0; e < S::PK; ++e) p.v[e] = page_of(key0 + vk + e);
    }
    return p;
  };
  // Address of a lane's piece of a key of page `page` (the pool's first slot where that is none).  Strides are
  // counted in 16-byte pieces: two 32-bit multiplications make the offset.
  auto place = [&](const char* base, const Stride16& t, int page, int key) -> const char* {
    const bool ok = (uint32_t)page < (uint32_t)a.table.num_pages;
    const int slot = key - fast_quot(a.table.page, key) * a.table.page.d;
    const uint64_t off = (uint64_t)(uint32_t)(ok ? page : 0) * t.page + (uint64_t)(uint32_t)(ok ? slot : 0) * t.slot;
    return base + (off << 4);
  };

  Tile<T, D> t;
  auto load_k = [&](const Pages& pg, int key0) {
#pragma unroll
    for (int i = 0; i < S::KSUB; ++i) {
      const char* p;
      if constexpr (OCT) p = place(kbase, ka.kst, pg.k[0], key0 + kk) + 4 * i * ((uint64_t)ka.kst.slot << 4);
      else p = place(kbase, ka.kst, pg.k[i], key0 + kk + 4 * i);
#pragma unroll
      for (int j = 0; j < S::KCH; ++j) t.k[i][j] = *(const u32x4*)(p + 64 * j);
    }
  };
  auto load_v = [&](const Pages& pg, int key0) {
    const char* p0;
    t.there = 0;
    if constexpr (OCT) {
      p0 = place(vbase, ka.vst, pg.v[0], key0 + vk);
      t.there = (uint32_t)pg.v[0] < (uint32_t)a.table.num_pages ? (1u << min(max(k_hi - (key0 + vk), 0), S::PK)) - 1u : 0u;
    }
#pragma unroll
    for (int e = 0; e < S::PK; ++e) {
      const char* p;
      if constexpr (OCT) {
        p = p0 + e * ((uint64_t)ka.vst.slot << 4);
      } else {
        const int page = pg.v[e];
        p = place(vbase, ka.vst, page, key0 + vk + e);
        t.there |= ((uint32_t)page < (uint32_t)a.table.num_pages ? 1u : 0u) << e;
      }
      if constexpr (BF && S::VW == 4) {
        const u32x4 z = *(const u32x4*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) t.v[e][i] = z[i];
      } else if constexpr (BF) {
        const u32x2 z = *(const u32x2*)p;
        t.v[e][0] = z[0];
        t.v[e][1] = z[1];
      } else {
#pragma unroll
        for (int f = 0; f < S::VP; ++f) {
          const u32x4 z = *(const u32x4*)(p + 256 * f);
#pragma unroll
          for (int i = 0; i < 4; ++i) t.v[e][4 * f + i] = z[i];
        }
      }
    }
  };

  constexpr int STEP = kWaves * S::KT;
  Pages pn;  // of the tile after the one that is loaded
  // Q^T: a thread brings (and rotates) 8 elements at a time, QN times
  constexpr int QN = (ROWS * (D / 8) + kThreads - 1) / kThreads;
  constexpr int QW = BF ? 1 : 2;  // 16-byte pieces of 8 elements
  u32x4 q_own[QN][QW], q_other[QN][QW];
  int col_pos[NT], rope_pos;  // positions of the columns' tokens, and of the block's token that this wavefront turns first
  // The next run of the share, with its first tile on the way; false when the share is done.
  auto begin = [&]() -> bool {
    for (;;) {
      if (x >= x_end) return false;
      const int take = min(row_units + kRowCost - at_w, x_end - x);
      u0 = max(at_w - kRowCost, 0);
      u1 = max(at_w + take - kRowCost, 0);
      if (u1 > u0) break;
      x += take;  // (a row's cost alone)
      at_w += take;
    }
    h = fast_quot(ka.blocks, item);
    key0 = (u0 << ka.unit_shift) + wave * S::KT;
    k_hi = u1 == row_units ? len : u1 << ka.unit_shift;
    // a lane's piece of a K row: 16 bytes at 16 g of each 64; of a V row: 16 (8: bf16 of head_dim 64) at its share n
    kbase = (const char*)((const T*)a.kc.ptr + h * a.kc.sh) + 16 * g;
    vbase = (const char*)((const T*)a.vc.ptr + h * a.vc.sh) + (BF ? 4 * S::VW : 16) * n;
    table = a.table.ptr + b * a.table.stride;
    const Pages pg = pages(key0);
    pn = pages(key0 + STEP);
    // (all that the run needs before its first scores is asked for ahead of the tile, which it would wait for otherwise)
    const int32_t* pos_b = a.positions + b * a.pos_stride;
    const int r0 = (item - h * ka.row_blocks) * ROWS;
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) col_pos[ct] = pos_b[fast_quot(ka.group, min(r0 + 16 * ct + n, ka.rows - 1))];
    rope_pos = pos_b[min(fast_quot(ka.group, r0) + wave, a.tokens - 1)];
#pragma unroll
    for (int i = 0; i < QN; ++i) {
      const int e = tid + i * kThreads, rl = e / (D / 8), d0 = e % (D / 8) * 8;
      const int r = min(r0 + rl, ka.rows - 1), tk = fast_quot(ka.group, r);
      const T* src = (const T*)a.q.ptr + b * a.q.sb + (h * group + (r - tk * group)) * a.q.sh + tk * a.q.ss;
      const int half = a.rope.rot / 2;
      const bool turns = rope && d0 < a.rope.rot;
      const T* other = src + (turns && !a.rope.interleaved ? (d0 < half ? d0 + half : d0 - half) : d0);
#pragma unroll
      for (int f = 0; f < QW; ++f) {
        q_own[i][f] = *(const u32x4*)((const char*)(src + d0) + 16 * f);
        if (QP == 3 || !BF) q_other[i][f] = *(const u32x4*)((const char*)other + 16 * f);
      }
    }
    load_k(pg, key0);
    load_v(pg, key0);
    return true;
  };
  bool busy = begin();
  bool first_run = true;

  while (busy) {
    const int r0 = (item - h * ka.row_blocks) * ROWS;  // the first row of the block
    const int32_t* pos_b = a.positions + b * a.pos_stride;

    // ---- Q^T to LDS, rotated: a lane forms its plane's cosine and sine of a token, for all heads
    const int t_first = fast_quot(ka.group, r0);  // of the block's tokens
    if (rope) {
      const int t_last = fast_quot(ka.group, min(r0 + ROWS, ka.rows) - 1);
      if (lane < a.rope.rot / 2) {
        for (int tk = t_first + wave; tk <= t_last; tk += kWaves) {
          float co, si;
          turn_cos_sin(rate, tk == t_first + wave ? rope_pos : pos_b[tk], co, si);
          sh.cs[tk - t_first][lane] = make_float2(co * a.rope.scale, si * a.rope.scale);
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < QN; ++i) {
      const int e = tid + i * kThreads, rl = e / (D / 8), d0 = e % (D / 8) * 8;
      if (rl >= ROWS) break;
      const bool turns = rope && d0 < a.rope.rot;
      const float2* cs = sh.cs[fast_quot(ka.group, min(r0 + rl, ka.rows - 1)) - t_first];
      if constexpr (BF) {
        const int j = d0 / 32, at = d0 % 32 / 8 * 16 + rl % 16;
        if constexpr (QP == 3) {
          float y[8], z[8];
          unpack8(q_own[i], y);
          unpack8(q_other[i], z);
          if (turns) rotate8(a.rope, cs, d0, y, z);
          bf16x8 z3[3];
          split3(y, z3);
#pragma unroll
          for (int part = 0; part < QP; ++part) sh.q[part][rl / 16][j][at] = __builtin_bit_cast(u32x4, z3[part]);
        } else {
          sh.q[0][rl / 16][j][at] = q_own[i][0];
        }
      } else {
        const int j = d0 / 16, at = d0 % 16 / 4 * 16 + rl % 16;
        float y[8], z[8];
        unpack8(q_own[i], y);
        unpack8(q_other[i], z);
        if (turns) rotate8(a.rope, cs, d0, y, z);
#pragma unroll
        for (int f = 0; f < 2; ++f)
          sh.q[0][rl / 16][j][at + 16 * f] = u32x4{__float_as_uint(y[4 * f]), __float_as_uint(y[4 * f + 1]),
                                                   __float_as_uint(y[4 * f + 2]), __float_as_uint(y[4 * f + 3])};
      }
    }

    // ---- the columns: rows r0 + 16 ct + n, the last key each sees.  Keys below `even` are seen alike by all live rows
    // (where no row is live, none matters): with one token a sequence, all of them.
    int last[NT], token[NT];
    int even = k_hi;
    if (a.tokens > 1) {
      int least = 0x7fffffff;
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) {
        token[ct] = fast_quot(ka.group, min(r0 + 16 * ct + n, ka.rows - 1));
        last[ct] = min(col_pos[ct], ka.capacity - 1);
        if (last[ct] >= 0) least = min(least, last[ct]);
      }
      least = __builtin_amdgcn_readfirstlane(row_min(least));
      if (least < len - 1) even = min(k_hi, (least + 1) / S::KT * S::KT);
    }
    __syncthreads();

    f32x4 acc[NT][NA];
#pragma unroll
    for (int ct = 0; ct < NT; ++ct)
#pragma unroll
      for (int i = 0; i < NA; ++i) acc[ct][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m[NT], l[NT];
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) m[ct] = -INFINITY, l[ct] = 0.f;

    // S^T of a column tile: element e is key key0 + PK g + e of the lane's column
    auto scores = [&](int ct, int at, float (&s)[S::PK]) {
      f32x4 y[S::KSUB * SUMS];
#pragma unroll
      for (int i = 0; i < S::KSUB * SUMS; ++i) y[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int part = QP - 1; part >= 0; --part)
#pragma unroll
        for (int j = 0; j < S::KCH; ++j) {
          const u32x4 q = sh.q[part][ct][j][at];
#pragma unroll
          for (int i = 0; i < S::KSUB; ++i) {
            if constexpr (BF) {
              y[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[i][j]),
                                                             __builtin_bit_cast(bf16x8, q), y[i], 0, 0, 0);
            } else {
#pragma unroll
              for (int f = 0; f < 4; ++f)
                y[f % SUMS] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.k[i][j][f]), __uint_as_float(q[f]),
                                                                   y[f % SUMS], 0, 0, 0);
            }
          }
        }
      if constexpr (SUMS == 4) y[0] = (y[0] + y[1]) + (y[2] + y[3]);
      if constexpr (SUMS == 2) y[0] += y[1];
#pragma unroll
      for (int i = 0; i < S::KSUB; ++i)
#pragma unroll
        for (int f = 0; f < 4; ++f) s[4 * i + f] = y[i][f];
    };

    // running maximum and sum; s becomes P
    auto softmax = [&](int ct, float (&s)[S::PK]) {
      float mx = s[0];
#pragma unroll
      for (int e = 1; e < S::PK; ++e) mx = fmaxf(mx, s[e]);
      mx = column_max(mx);
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

    // P^T as the operand of the second product (bf16: in three parts, fp32 whole)
    struct Weights {
      bf16x8 part[3];
      float p[S::PK];
    };
    auto weights = [&](const float (&p)[S::PK]) -> Weights {
      Weights w;
      if constexpr (BF) {
        split3(p, w.part);
      } else {
#pragma unroll
        for (int e = 0; e < S::PK; ++e) w.p[e] = p[e];
      }
      return w;
    };
    // y + V^T P^T of accumulator i, the bits outside `keep` taken as 0.  Element f of the
    // lane: column n, feature (4 g + f) D / 16 + i (bf16), 64 (i / 4) + 4 (4 g + f) + i % 4 (fp32)
    auto product = [&](const Weights& w, int i, f32x4 y, const uint32_t (&keep)[4], const uint32_t (&take)[2]) -> f32x4 {
      if constexpr (BF) {
        u32x4 z;
#pragma unroll
        for (int f = 0; f < 4; ++f)
          z[f] = keep[f] & __builtin_amdgcn_perm(t.v[2 * f + 1][i / 2], t.v[2 * f][i / 2], take[i % 2]);
        const bf16x8 vt = __builtin_bit_cast(bf16x8, z);
#pragma unroll
        for (int part = 2; part >= 0; --part) y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, w.part[part], y, 0, 0, 0);
        return y;
      } else {
#pragma unroll
        for (int e = 0; e < S::PK; ++e)
          y = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[e][i] & keep[e]), w.p[e], y, 0, 0, 0);
        return y;
      }
    };

    constexpr uint32_t kTake[2] = {0x05040100u, 0x07060302u};  // the low and the high halves of two dwords

    // the bits of V's operands that belong to the keys in `seen`
    auto mask = [&](uint32_t seen, uint32_t (&keep)[4]) {
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        if constexpr (BF) keep[f] = (seen >> 2 * f & 1 ? 0xffffu : 0u) | (seen >> (2 * f + 1) & 1 ? 0xffff0000u : 0u);
        else keep[f] = seen >> f & 1 ? ~0u : 0u;
      }
    };

    // Tiles that all live rows see alike.  A tile's K registers take the next tile's keys as soon as its scores are
    // formed, its V registers after the second product, so that loads are always in flight; pages are looked up
    // two tiles ahead (loads return in order: a look-up behind a tile's loads would wait for them).
    int at = lane;
    for (; key0 < even; key0 += STEP) {
      asm volatile("" : "+v"(at));  // (the reads of Q^T stay in the loop: kept in registers, they would spill)
      float s[NT][S::PK];
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) scores(ct, at, s[ct]);
      __builtin_amdgcn_sched_barrier(0);  // (the next keys take the registers of these)
      const Pages pg = pn;
      pn = pages(key0 + 2 * STEP);
      load_k(pg, key0 + STEP);
      // (what stands in slots that no row sees may be anything: always masked, which the loads' time hides)
      uint32_t keep[4];
      mask(t.there, keep);
      Weights w[NT];
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) {
#pragma unroll
        for (int e = 0; e < S::PK; ++e) s[ct][e] = t.there >> e & 1 ? s[ct][e] : -INFINITY;
        softmax(ct, s[ct]);
        w[ct] = weights(s[ct]);
      }
#pragma unroll
      for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int ct = 0; ct < NT; ++ct) acc[ct][i] = product(w[ct], i, acc[ct][i], keep, kTake);
      __builtin_amdgcn_sched_barrier(0);  // (as above, for V)
      load_v(pg, key0 + STEP);
    }
    // The keys near the new tokens, whose rows see different ones: one that a token does not see must not
    // reach its output even as 0 times whatever V holds.
    for (; key0 < k_hi; key0 += STEP) {
      const int lane_key = key0 + vk;
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) {
        float s[S::PK];
        scores(ct, lane, s);
#pragma unroll
        for (int e = 0; e < S::PK; ++e) s[e] = (t.there >> e & 1) && lane_key + e <= last[ct] ? s[e] : -INFINITY;
        softmax(ct, s);
        const Weights w = weights(s);
        const int t_lo = fast_quot(ka.group, min(r0 + 16 * ct, ka.rows - 1));
        const int t_hi = fast_quot(ka.group, min(r0 + 16 * ct + 15, ka.rows - 1));
        for (int tk = t_lo; tk <= t_hi; ++tk) {
          const int end = max(min(pos_b[tk], ka.capacity - 1), -1) + 1;  // the token's keys
          const uint32_t seen = t.there & ((1u << min(max(end - lane_key, 0), S::PK)) - 1u);
          uint32_t keep[4];
          mask(seen, keep);
          uint32_t take[2] = {kTake[0], kTake[1]};
          asm volatile("" : "+s"(take[0]), "+s"(take[1]));  // (V is transposed here each time: kept for all tokens, it would spill)
#pragma unroll
          for (int i = 0; i < NA; ++i) {
            __builtin_amdgcn_sched_barrier(0);  // (one at a time: side by side they would spill)
            const f32x4 o = product(w, i, f32x4{0.f, 0.f, 0.f, 0.f}, keep, take);
            if (token[ct] == tk) acc[ct][i] += o;
          }
        }
      }
      if (key0 + STEP < k_hi) {
        load_k(pn, key0 + STEP);
        load_v(pn, key0 + STEP);
        pn = pages(key0 + 2 * STEP);
      }
    }

    // ---- the next run, its first tile in flight under this one's end
    const int cur_b = b, cur_item = item, cur_h = h;
    bool dead[NT];  // (a token at a negative position: no weight, whatever its columns held)
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) dead[ct] = col_pos[ct] < 0;
    const bool opens = u0 == 0, whole = opens && u1 == row_units;
    const int row_last = x - at_w + row_units + kRowCost - 1;  // the row's last unit
    const int done = u1 + kRowCost - at_w;
    x += done;
    at_w += done;
    if (u1 == row_units) {
      at_w = 0;
      if (++item == items) {
        item = 0;
        ++b;
        if (x < x_end) {
          len = __builtin_amdgcn_readfirstlane(length_of(ka, b));
          row_units = units_of(ka, len);
        }
      }
    }
    busy = begin();

    // ---- the wavefronts' results together
    const int nrows = min(ROWS, ka.rows - r0);
    __syncthreads();  // sh.q is read
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) {
      l[ct] = column_sum(l[ct]);
      const int col = 16 * ct + n;
      if (g == 0) {
        sM[wave][col] = dead[ct] ? -INFINITY : m[ct];
        sL[wave][col] = dead[ct] ? 0.f : l[ct];
      }
      if (col < nrows)
#pragma unroll
      for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const int d = BF ? (4 * g + f) * NA + i : 64 * (i / 4) + 4 * (4 * g + f) + i % 4;
          sh.o[wave][col][d] = acc[ct][i][f];
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
        o += wgt * *(const f32x4*)&sh.o[i][rl][d];
      }
      if (!whole) {
        *(f32x4*)(ka.part_o + ((int64_t)slot * ROWS + rl) * D + d) = o;
        if (d == 0) ka.part_ml[(int64_t)slot * ROWS + rl] = make_float2(mx, sum);
        continue;
      }
      const int r = r0 + rl, tk = fast_quot(ka.group, r), hq = cur_h * group + (r - tk * group);
      const bool none = sum == 0.f;
      const float inv = none ? 0.f : 1.f / sum;
      T* out = (T*)a.o + cur_b * a.osb + hq * a.osh + tk * a.oss + d;
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const float y = none ? 0.f : o[f] * inv;
        if constexpr (BF) ((__bf16*)out)[f] = (__bf16)y;
        else out[f] = y;
      }
      if (a.lse != nullptr && d == 0)
        a.lse[((int64_t)cur_b * a.heads_q + hq) * a.tokens + tk] =
            none ? -INFINITY : ((mx == -INFINITY ? 0.f : mx * c) + __log2f(sum)) * kLn2;
    }
    if (ka.join && opens && tid == 0)
      ka.record[(int64_t)cur_b * items + cur_item] = whole ? make_int2(-1, -1) : make_int2(slot, deal.owner(row_last));
    if (!busy) break;
    first_run = false;
    __syncthreads();  // sh.o is read
  }
}

// Rows whose keys several workgroups shared: their partial results, in the order of the keys.  A workgroup joins JR
// rows of an item, a wavefront forming the weights of a row (or part of one: all four then form the same); a thread sums
// 4 features over the parts grp, grp + GRP, ..  Four rows a workgroup keep a large batch's launch short, one row leaves
// fewer parts to each thread where the call has few rows (a token after 131072 tokens, 32 rows of 64 parts: 6.9 -> 4.8 us).
constexpr int kJoinThreads = 256;
template <typename T, int D, int JR>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(KernelArgs ka, int rows_block) {
  constexpr int V4 = D / 4, GRP = kJoinThreads / (V4 * JR), AHEAD = 8, OWN = kWorkers / kWave;
  __shared__ float sW[JR][kWorkers];
  __shared__ float2 sT[JR];
  __shared__ __attribute__((aligned(16))) float sO[GRP][JR][D];
  const PagedArgs& a = ka.a;
  asm volatile("" ::"s"(a.osb), "s"(a.lse), "s"(a.batch), "s"(ka.rows), "s"(ka.part_o));  // (as in the kernel before)
  const int2 rec = ka.record[blockIdx.x];
  if (rec.x < 0) return;
  const int items = a.heads_kv * ka.row_blocks;
  const int b = blockIdx.x / (uint32_t)items, item = blockIdx.x - b * items;
  const int h = fast_quot(ka.blocks, item), rb = item - h * ka.row_blocks;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int nrows = min(rows_block, ka.rows - rb * rows_block);
  const int w0 = rec.x / 2, parts = rec.y - w0 + 1;
  auto slot = [&](int p, int rl) { return (int64_t)(p == 0 ? rec.x : 2 * (w0 + p)) * rows_block + rl; };
  const float c = ka.scale_log2;

  // the first parts are on their way while the weights are formed
  const int wrow = wave % JR;
  const int row = min((int)blockIdx.y * JR + wrow, nrows - 1);
  float2 ml[OWN];
#pragma unroll
  for (int i = 0; i < OWN; ++i)
    if (i * kWave < parts) ml[i] = ka.part_ml[slot(min(lane + i * kWave, parts - 1), row)];
  const int d = tid % V4 * 4, jr = tid / V4 % JR, grp = tid / (V4 * JR);
  const int rl = min((int)blockIdx.y * JR + jr, nrows - 1);
  auto part = [&](int p) { return *(const f32x4*)(ka.part_o + slot(p, rl) * D + d); };
  f32x4 y[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) y[i] = part(min(grp + i * GRP, parts - 1));

  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < OWN; ++i)
    if (i * kWave < parts) mx = fmaxf(mx, ml[i].x);
  mx = wave_max(mx);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < OWN; ++i)
    if (lane + i * kWave < parts) {
      const float wgt = ml[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[i].x - mx) * c);
      if (wave < JR) sW[wrow][lane + i * kWave] = wgt;
      sum += wgt * ml[i].y;
    }
  sum = wave_sum(sum);
  if (lane == 0 && wave < JR) sT[wrow] = make_float2(mx, sum);
  __syncthreads();

  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (grp + i * GRP < parts) o += sW[jr][grp + i * GRP] * y[i];
#pragma unroll 4
  for (int p = grp + AHEAD * GRP; p < parts; p += GRP) o += sW[jr][p] * part(p);
  *(f32x4*)&sO[grp][jr][d] = o;
  __syncthreads();
  if (grp != 0 || (int)blockIdx.y * JR + jr >= nrows) return;
#pragma unroll
  for (int i = 1; i < GRP; ++i) o += *(const f32x4*)&sO[i][jr][d];
  mx = sT[jr].x;
  sum = sT[jr].y;
  const int r = rb * rows_block + rl, t = fast_quot(ka.group, r), hq = h * ka.group.d + (r - t * ka.group.d);
  const bool none = sum == 0.f;
  T* out = (T*)a.o + b * a.osb + hq * a.osh + t * a.oss + d;
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const float z = none ? 0.f : o[f] / sum;
    if constexpr (sizeof(T) == 2) ((__bf16*)out)[f] = (__bf16)z;
    else out[f] = z;
  }
  if (a.lse != nullptr && d == 0)
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
    if (k.a.rope.freq) e = nt == 2 ? launch<T, D, 2, 3>(k, grid, s) : launch<T, D, 1, 3>(k, grid, s);
    else e = nt == 2 ? launch<T, D, 2, 1>(k, grid, s) : launch<T, D, 1, 1>(k, grid, s);
  } else {
    e = nt == 2 ? launch<T, D, 2, 1>(k, grid, s) : launch<T, D, 1, 1>(k, grid, s);
  }
  if (e != hipSuccess || !k.join) return e;
  const int64_t all = (int64_t)k.a.batch * k.a.heads_kv * k.row_blocks;
  const int rows = std::min(k.rows, 16 * nt);
  if (all * rows <= 2 * kWorkers)
    paged_join_kernel<T, D, 1><<<dim3((unsigned)all, (unsigned)rows), kJoinThreads, 0, s>>>(k, 16 * nt);
  else
    paged_join_kernel<T, D, 4><<<dim3((unsigned)all, (unsigned)((rows + 3) / 4)), kJoinThreads, 0, s>>>(k, 16 * nt);
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
  const int piece = a.bf16 ? 8 : 4;
  k.kst = {(uint32_t)(a.kc.sp / piece), (uint32_t)(a.kc.ss / piece)};
  k.vst = {(uint32_t)(a.vc.sp / piece), (uint32_t)(a.vc.ss / piece)};
  k.group = fast_div(p.group);
  k.blocks = fast_div(p.row_blocks);
  k.rows = p.rows;
  k.row_blocks = p.row_blocks;
  k.capacity = a.table.max_pages * a.table.page.d;  // (at most 2^30: no sum of keys overflows)
  const int64_t items = (int64_t)a.heads_kv * p.row_blocks;
  const int64_t rows = items * a.batch;  // a KV head's, as the workgroups take them
  k.join = k.capacity > (a.bf16 ? kWholeKeys : kWholeKeys / 2) * (rows >= 128 && rows <= kWorkers ? 2 : 1);
  // a unit is a tile for each wavefront; a whole row where rows are not split, and more where the weights of all units
  // would not stay below 2^30
  k.unit_shift = a.bf16 ? 7 : 6;
  static_assert(kWaves == 4, "128 keys of bf16, 64 of fp32");
  auto units = [&]() -> int64_t { return ((int64_t)k.capacity + ((int64_t)1 << k.unit_shift) - 1) >> k.unit_shift; };
  while ((!k.join && units() > 1) || (units() + 2) * rows > (1 << 30)) ++k.unit_shift;
  k.scale_log2 = a.scale * kLog2e;
  char* ws = (char*)a.workspace;
  k.record = (int2*)ws;
  k.part_ml = (float2*)(ws + p.ml);
  k.part_o = (float*)(ws + p.o);
  const dim3 grid((unsigned)std::min((int64_t)kWorkers, units() * rows));
  if (a.bf16) return a.head_dim == 128 ? launch_typed<uint16_t, 128>(k, p.nt, grid, s) : launch_typed<uint16_t, 64>(k, p.nt, grid, s);
  return a.head_dim == 128 ? launch_typed<float, 128>(k, p.nt, grid, s) : launch_typed<float, 64>(k, p.nt, grid, s);
}

}  // namespace seer
