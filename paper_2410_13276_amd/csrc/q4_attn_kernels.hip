// q4_attn_kernels.hip -- attention of new tokens over a paged cache held in 4 bits.
//
// As over a cache of values (paged_attn_kernels.hip) the rows of a KV group are the columns of S^T = K Q^T and O^T = V^T P^T, and
// the units of all sequences' keys are dealt out evenly to the workgroups.  What differs is that a key is 36 to 80 bytes and
// has to be opened: at 5 bits an element HBM brings about 8e12 elements a second, for which the
// vector units have some 4 operations each.  So codes enter the matrix products as they are, and steps and
// middles are applied to what comes out or goes in:
//
//   q . k = sum over groups g of step_g sum_{d in g} q_d (c_d - 7.5) + mid_g sum_{d in g} q_d
//   o_d   = sum over keys t of (p_t step_tg) (c_td - 7.5) + p_t mid_tg
//
// Opening.  Bits 3 to 6 of a bf16 number in [1, 2) are a code: 1 + c / 16, one shift and one three-input boolean operation
// for two codes.  The 1 is taken out again in fp32, at the sums' starting values, and half of the codes (4 of 8) enter
// complemented, 1 + (15 - c) / 16, their factors negated: with u = 1.46875 = 1 + 7.5 / 16 either is u +- (c - 7.5) / 16, so that
// what has to be taken out is u times a sum of terms of both signs, which stays as small as the result.  (All of one
// sign, the second product's sums would be 5 to 100 times the result and carry their rounding into it.)  Where the output is fp32, codes
// are looked up as (c - 7.5) / 16 instead, exactly, and nothing is taken out (1000 keys: o 1.6e-7 to 2.5e-7 off in the 2-norm, and 7e-7 to 1.1e-6
// as above, 2e-6 to 3e-6 where one element of each group is far off; 65536 tokens of 32 / 8 heads of 128 34 us, and 30).
//
// Rows.  A step belongs to a group, so that a group's products may not run into another's sum.  Where a block has
// few rows (16 / (D / group) at most), the 16 rows of the products' other operand are pairs of row and group: Q is 0 but in
// the pair's group, which gives S by groups in one accumulator, the groups of a row in one lane, which adds them up;
// and P^T in column (r, g) is p step_g, of which the outputs of group g take theirs.  With more rows the pairs are rows alone (or
// of two groups), and the groups are done one after the other.  Weights go from the lanes of their keys to those of the second
// product's operand through the LDS, so that no weight is formed twice.
//
// A wavefront takes 64 keys at a time.  K's codes come to registers as the operand wants them (16 bytes of one
// key a lane); V's go through the wavefront's own LDS and come back transposed (ds_read_b64_tr_b4: 16 keys of
// one channel a lane); so do both params.  Where pages hold whole aligned runs of 16 keys, a lane looks up a run's address
// for all.
//
// Precision: fp32 statistics and sums.  A q that is rotated here, or fp32, enters in three bf16 parts, which hold fp32 whole (two,
// rounded to nearest, left the log-sum-exp 1e-6 of itself off where this leaves 1e-7), and so does p step where the output is
// fp32; where it is bf16, in two, 2^-18 of it off at most, where the output's own rounding is 2^-9.
//
// Measured (bf16, one MI355X): 32 / 8 heads of 128 in groups of 32, a token after 131072 tokens 42 us + 4 of the join, for 168 MB
// (4e12 bytes a second while it runs; a kernel that only reads reaches 6.2e12); 64 sequences of 200 to 16000 tokens 77 + 4.5 for
// 285 MB.  What bounds it is latency, a tile's chain of dependent steps at two wavefronts a SIMD first (without any loads it takes
// 34 us of 43, without products 39), its loads beside it (one tile, 10 KB, in flight a wavefront; a second in registers spills: 79
// us); the vector units issue 0.46 of the time, the matrix units work 0.2.  About 9 us are a run's beginning (positions, table,
// tile, one after the other) and end.  With 16 rows and more a tile's own chain is what takes long, scores, weights and factors of
// two or four phases: 28 rows of 4 heads over 93643 tokens in groups of 64 46 us for 54 MB.
#include <algorithm>
#include <type_traits>

#include "cache.h"
#include "paged_join.h"
#include "q4_open.h"

namespace seer {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kKeys = 64;      // of a tile
// Rows with room for so many keys are not split, which saves the joining launch (32 / 8 heads of 128, 500 keys in room for 512: a
// sequence 9.3 us against 12.6 split, 64 of them 13.8 against 15.3; 1000 in 1024: a sequence 13.2 whole, 12.6 split).
constexpr int kWholeKeys = 512;

struct PoolStrides {  // of codes in 16-byte pieces, of params in rows of them
  uint32_t page, slot, ppage, pslot;
};

struct KernelArgs {
  Q4AttnArgs a;
  PoolStrides kst, vst;
  int rows, row_blocks;      // G tokens, blocks of ROWS rows
  FastDiv group, blocks;     // by G and row_blocks
  int capacity;              // tokens that a table row has room for
  int unit_shift;            // log2 of the keys per unit
  bool join;                 // rows may be split: records are written for the second launch
  float scale_log2;          // of a score / 16
  int2* record;              // [batch heads_kv row_blocks] first slot and last workgroup of a split row, or -1
  float2* part_ml;           // [2 kWorkers][ROWS] maximum and sum
  float* part_o;             // [2 kWorkers][ROWS][D]
};

// Keys that the tokens of a sequence see at most.
__device__ __forceinline__ int length_of(const KernelArgs& k, int b) {
  int len = 0;
  const int32_t* p = k.a.q.positions + b * k.a.q.pos_stride;
  for (int s = 0; s < k.a.q.tokens; ++s) len = max(len, min(p[s], k.capacity - 1) + 1);
  return len;
}
__device__ __forceinline__ int units_of(const KernelArgs& k, int len) {
  return max(1, (len + (1 << k.unit_shift) - 1) >> k.unit_shift);
}

typedef __attribute__((ext_vector_type(2))) int i32x2;

// Largest and sum of a row of 16 lanes, for all of them.
__device__ __forceinline__ float row_max(float x) {
  auto with = [&](int y) { x = fmaxf(x, __int_as_float(y)); };
  with(dpp<0xb1>(0, __float_as_int(x)));   // quad_perm 1 0 3 2
  with(dpp<0x4e>(0, __float_as_int(x)));   // quad_perm 2 3 0 1
  with(dpp<0x141>(0, __float_as_int(x)));  // row_half_mirror
  with(dpp<0x140>(0, __float_as_int(x)));  // row_mirror
  return x;
}
__device__ __forceinline__ float row_sum(float x) {
  x = dpp_add<0xb1>(x);
  x = dpp_add<0x4e>(x);
  x = dpp_add<0x141>(x);
  return dpp_add<0x140>(x);
}

// D: elements of a head.  NG: groups of a head.  PACK: of them, those that share the columns.  QP: bf16 parts of q (1: bf16
// as it is, 3: rotated, or fp32).
// RUN: pages hold whole aligned runs of 16 keys, whose rows lie within 2^30 bytes (a token after 131072 tokens, replayed from a
// graph: pages of 64 46 us, of 24, which are looked up key by key, 50, of 1 81).
template <typename T, int D, int NG, int PACK, int QP, bool RUN>
__global__ __launch_bounds__(kThreads, 2) void q4_attn_kernel(KernelArgs ka) {
  constexpr int ROWS = 16 / PACK, NPH = NG / PACK;
  constexpr int RV = 4 / PACK;         // rows whose scores a lane holds
  constexpr int NA = D / 16;           // accumulators: 16 channels each
  constexpr int QD = D / 32;           // dwords of a key's codes per lane
  constexpr int SIDE = 2;              // sums of the second product that are formed side by side
  constexpr int OSTR = D + 4;
  constexpr int PSTR = kKeys + 16 / RV;  // (rows of the weights fall on different banks)
  constexpr bool BF = sizeof(T) == 2;
  constexpr int PP = BF ? 2 : 3;       // bf16 parts of a weight times its step
  // fp32: what a tile adds is formed by itself and then added; bf16: the sums run on over the tiles, the factors' own
  // beside them (its rounding, 2^-9, hides what that leaves)
  constexpr bool RUNS = BF;
  auto open = [](uint32_t codes) {
    if constexpr (BF) return open8(codes);
    else return open8_centred(codes);
  };
  constexpr int kRowCost = 1;          // a row's beginning and end, in units
  constexpr int PIECES = D / 8;
  // with more phases than one, K's codes are brought into the order of their channels, so that a step of the product has
  // the channels of one group only
  constexpr bool ALIGNED = NPH > 1 && PACK == 1;
  // of four phases the sums of Q's groups are read from the LDS each time (28 rows over 8 x 4096 tokens, groups of 32:
  // held, 55.1 us, with 96 spills; read, 39.3)
  constexpr bool SUMS_HELD = NPH < 4;
  constexpr bool HELD = NPH == 1 && QP * QD <= 8;  // Q stays in registers
  using Piece = std::conditional_t<QD == 4, u32x4, u32x2>;  // a quarter of a row of codes
  __shared__ union {
    struct {
      u32x4 q[QP][QD][kWave];          // 8 elements in open8's order, 4 to 7 negated, as the lanes read them
      float2 sum[ROWS][NG];            // of a row's elements in a group: as above, and all / 16
      float2 cs[ROWS][D / 2];
      struct {
        Piece v[kKeys][4];
        float ks[kKeys][NG], km[kKeys][NG];                    // steps and middles: key, group
        float vs[4][NG + 1][16], vm[4][NG + 1][16];            // run, group, key
        float p[ROWS][PSTR];
        float alpha[ROWS];
      } w[kWaves];
    };
    float o[kWaves][ROWS][OSTR];
  } sh;
  __shared__ float sM[kWaves][ROWS], sL[kWaves][ROWS];

  const QueryArgs& a = ka.a.q;
  const CacheArgs& ca = a.cache;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane % 16, j = lane / 16;
  const int gp = n % PACK, row = n / PACK;  // of the operand Q's row n, and of column n of the second product
  const int items = ca.heads_kv * ka.row_blocks;  // rows of a sequence
  const int group = ka.group.d;
  const float c = ka.scale_log2;
  const bool rope = QP != 1 && a.rope.freq != nullptr;
  const double freq = (rope ? a.rope.freq : (const double*)ca.k.data)[rope ? min(lane, a.rope.rot / 2 - 1) : 0];

  // ---- this workgroup's share (every wavefront works it out by itself)
  const int share = (a.batch + kWave - 1) / kWave;  // sequences per lane
  const int b_lo = min(lane * share, a.batch), b_hi = min(b_lo + share, a.batch);
  int mine = 0, my_len = 0;
  for (int i = b_lo; i < b_hi; ++i) {
    my_len = length_of(ka, i);
    mine += units_of(ka, my_len) + kRowCost;
  }
  const int upto = wave_prefix(mine);
  const TurnRate rate = turn_rate(freq);
  const Deal deal((uint32_t)(__builtin_amdgcn_readlane(upto, kWave - 1) * items), gridDim.x);
  if (blockIdx.x >= (uint32_t)deal.workers) return;
  const int w = share_of(ca.k, a.batch, blockIdx.x, (int)deal.workers);
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

  // ---- a run of one row's units [u0, u1)
  int u0, u1, h, key0, k_hi, last_page;
  const char *kbase, *vbase;
  const uint32_t *kpbase, *vpbase;
  const int32_t* table;

  // K: lane n of sub-tile i is key 16 i + n, a quarter of its row; V's codes: load i brings a quarter of token 16 i + lane / 4;
  // params: token `lane`.  Where pages hold whole aligned runs, a lane looks up the run of token `lane` alone.
  struct At {
    int page;
    uint32_t slot;
  };
  struct Pages {
    At k[RUN ? 1 : 4], v[RUN ? 1 : 4], p;
  };
  // A key's page, as the table has it, and slot.  (A key past the run is taken to be on its last one's page: no branch.
  // Nothing is done with what is found until it is used, a tile later, as it would be waited for here.)
  auto page_of = [&](int key) -> At {
    const int i = fast_quot(ca.table.page, key);
    return {table[min(i, last_page)], (uint32_t)(key - i * ca.table.page.d)};
  };
  auto pages = [&](int key0) -> Pages {
    Pages p;
    if constexpr (!RUN) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p.k[i] = page_of(key0 + 16 * i + n);
        p.v[i] = page_of(key0 + 16 * i + lane / 4);
      }
    }
    p.p = page_of(key0 + (RUN ? 16 * j : lane));
    return p;
  };
  // Offset of a key's row in units of the strides' (the pool's first page where it has none).
  auto has_page = [&](int page) { return (uint32_t)page < (uint32_t)ca.table.num_pages; };
  auto offset = [&](const At& s, uint32_t page, uint32_t slot) {
    return (uint64_t)(has_page(s.page) ? (uint32_t)s.page : 0u) * page + (uint64_t)s.slot * slot;
  };
  // (a lane forms its run's, for all)
  auto of_run = [&](uint64_t off, int i) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(off >> 32), 16 * i) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)off, 16 * i);
  };

  Piece kq[4], vq[4];
  uint32_t kpq[NG], vpq[NG];
  bool there;             // token `lane` exists
  // a lane's place within a run
  const uint32_t klane = (uint32_t)(n * (int)(RUN ? ca.k.ss : 0)) + sizeof(Piece) * j;
  const uint32_t vlane = (uint32_t)(lane / 4 * (int)(RUN ? ca.v.ss : 0)) + sizeof(Piece) * (lane % 4);
  // (past the caches: a token after 131072 tokens 42.7 -> 39.8 us, 64 mixed sequences 77.5 -> 72.1)
  auto past = [](const char* p) { return __builtin_nontemporal_load((const Piece*)p); };
  auto load_k = [&](const Pages& pg) {
    const uint64_t mine = RUN ? offset(pg.p, ka.kst.page, ka.kst.slot) << 4 : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      kq[i] = past(kbase + (RUN ? of_run(mine, i) : offset(pg.k[RUN ? 0 : i], ka.kst.page, ka.kst.slot) << 4) + klane);
  };
  auto load_v = [&](const Pages& pg, int key0) {
    const uint64_t mine = RUN ? offset(pg.p, ka.vst.page, ka.vst.slot) << 4 : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      vq[i] = past(vbase + (RUN ? of_run(mine, i) : offset(pg.v[RUN ? 0 : i], ka.vst.page, ka.vst.slot) << 4) + vlane);
    there = has_page(pg.p.page) && key0 + lane < k_hi;
    const At own = {pg.p.page, pg.p.slot + (RUN ? n : 0)};
    const uint32_t* kp = kpbase + offset(own, ka.kst.ppage, ka.kst.pslot) * NG;
    const uint32_t* vp = vpbase + offset(own, ka.vst.ppage, ka.vst.pslot) * NG;
    if constexpr (NG == 4) {
      const u32x4 y = *(const u32x4*)kp, z = *(const u32x4*)vp;
#pragma unroll
      for (int g = 0; g < 4; ++g) kpq[g] = y[g], vpq[g] = z[g];
    } else if constexpr (NG == 2) {
      const u32x2 y = *(const u32x2*)kp, z = *(const u32x2*)vp;
      kpq[0] = y[0], kpq[1] = y[1], vpq[0] = z[0], vpq[1] = z[1];
    } else {
      kpq[0] = kp[0], vpq[0] = vp[0];
    }
  };

  constexpr int STEP = kWaves * kKeys;
  Pages pn;  // of the tile after the one that is loaded
  // a thread's 8 elements of Q^T, and the others of their planes; positions of the column's token and of the block's token
  // that this wavefront turns first
  constexpr int QW = BF ? 1 : 2;
  u32x4 q_own[QW], q_other[QW];
  int col_pos, row_pos[RV], rope_pos = 0;
  static_assert(ROWS * PIECES <= kThreads, "one piece a thread");
  const int q_row = min(tid / PIECES, ROWS - 1), q_d0 = tid % PIECES * 8;
  const bool turns = rope && q_d0 < a.rope.rot;
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
    key0 = (u0 << ka.unit_shift) + wave * kKeys;
    k_hi = u1 == row_units ? len : u1 << ka.unit_shift;
    last_page = last_page_of(ca.table.page, k_hi);
    kbase = (const char*)ca.k.data + h * ca.k.sh;
    vbase = (const char*)ca.v.data + h * ca.v.sh;
    kpbase = ca.k.params + h * ca.k.psh;
    vpbase = ca.v.params + h * ca.v.psh;
    table = ca.table.ptr + b * ca.table.stride;
    const Pages pg = pages(key0);
    pn = pages(key0 + STEP);
    // (all that the run needs before its first scores is asked for ahead of the tile, which it would wait for otherwise)
    const int r0 = (item - h * ka.row_blocks) * ROWS;
    col_pos = a.positions[b * a.pos_stride + fast_quot(ka.group, min(r0 + row, ka.rows - 1))];
#pragma unroll
    for (int v = 0; v < RV; ++v)
      row_pos[v] = a.positions[b * a.pos_stride + fast_quot(ka.group, min(r0 + RV * j + v, ka.rows - 1))];
    if (rope) rope_pos = a.rope_positions[b * a.pos_stride + min(fast_quot(ka.group, r0) + wave, a.tokens - 1)];
    {
      const int r = min(r0 + q_row, ka.rows - 1), tk = fast_quot(ka.group, r), half = a.rope.rot / 2;
      const T* src = (const T*)a.q.ptr + b * a.q.sb + (h * group + (r - tk * group)) * a.q.sh + tk * a.q.ss;
      const T* other = src + (turns && !a.rope.interleaved ? (q_d0 < half ? q_d0 + half : q_d0 - half) : q_d0);
#pragma unroll
      for (int f = 0; f < QW; ++f) {
        q_own[f] = *((const u32x4*)(src + q_d0) + f);
        if (QP != 1) q_other[f] = *((const u32x4*)other + f);
      }
    }
    load_v(pg, key0);
    load_k(pg);
    return true;
  };
  bool busy = begin();
  bool first_run = true;

  while (busy) {
    const int r0 = (item - h * ka.row_blocks) * ROWS;  // the first row of the block

    // ---- Q^T to LDS, rotated: a lane forms its plane's cosine and sine of a token, for all heads
    const int t_first = fast_quot(ka.group, r0);  // of the block's tokens
    if (rope) {
      const int t_last = fast_quot(ka.group, min(r0 + ROWS, ka.rows) - 1);
      const int32_t* rpos_b = a.rope_positions + b * a.pos_stride;
      if (lane < a.rope.rot / 2) {
        for (int tk = t_first + wave; tk <= t_last; tk += kWaves) {
          float co, si;
          turn_cos_sin(rate, tk == t_first + wave ? rope_pos : rpos_b[tk], co, si);
          sh.cs[tk - t_first][lane] = make_float2(co * a.rope.scale, si * a.rope.scale);
        }
      }
      __syncthreads();
    }
    if (tid < ROWS * PIECES) {
      const int rl = q_row, d0 = q_d0;
      float y[8], z[8];
      unpack8(q_own, y);
      if (turns) {
        unpack8(q_other, z);
        rotate8(a.rope, sh.cs[fast_quot(ka.group, min(r0 + rl, ka.rows - 1)) - t_first], d0, y, z);
      }
      // sums over the group's pieces, which neighbours hold
      const float lo = (y[0] + y[1]) + (y[2] + y[3]), hi = (y[4] + y[5]) + (y[6] + y[7]);
      float sgn = lo - hi, all = lo + hi;
      sgn = dpp_add<0xb1>(sgn), all = dpp_add<0xb1>(all);
      sgn = dpp_add<0x4e>(sgn), all = dpp_add<0x4e>(all);
      if constexpr (D / NG == 64) sgn = dpp_add<0x141>(sgn), all = dpp_add<0x141>(all);
      if (d0 % (D / NG) == 0) sh.sum[rl][d0 / (D / NG)] = make_float2(sgn, all * 0.0625f);
#pragma unroll
      for (int e = 4; e < 8; ++e) y[e] = -y[e];
      const float s8[8] = {y[0], y[4], y[1], y[5], y[2], y[6], y[3], y[7]};
      bf16x8 parts[QP];
      split<QP>(s8, parts);  // (a bf16 q that is not rotated is its own first part)
      // lane (quad of channels, operand row): 0 in the pairs of other groups, where the pairs hold all groups
#pragma unroll
      for (int part = 0; part < QP; ++part)
#pragma unroll
        for (int g = 0; g < PACK; ++g) {
          const bool own = NPH > 1 || d0 / (D / NG) == g;
          (ALIGNED ? sh.q[part][tid % PIECES / 4][16 * (tid % PIECES % 4) + rl]
                   : sh.q[part][tid % PIECES % QD][16 * (tid % PIECES / QD) + rl * PACK + g]) =
              own ? __builtin_bit_cast(u32x4, parts[part]) : u32x4{0, 0, 0, 0};
        }
    }
    // the last key that the lane's column, and its rows, see; and that all rows do
    const int last = min(col_pos, ka.capacity - 1);
    int sees[RV], least = last;
#pragma unroll
    for (int v = 0; v < RV; ++v) sees[v] = min(row_pos[v], ka.capacity - 1);
    least = __builtin_amdgcn_readfirstlane(row_min(least));
    __syncthreads();

    const int quad_group = j * NG / 4;
    u32x4 q[HELD ? QP : 1][QD];
    if constexpr (HELD)
#pragma unroll
      for (int part = 0; part < QP; ++part)
#pragma unroll
        for (int i = 0; i < QD; ++i) q[part][i] = sh.q[part][i][lane];
    f32x4 from[SUMS_HELD ? NPH : 1], all[SUMS_HELD ? NPH : 1];  // of the lane's pairs of row and group
    if constexpr (SUMS_HELD)
#pragma unroll
    for (int ph = 0; ph < NPH; ++ph)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float2 y = sh.sum[RV * j + r / PACK][ph * PACK + r % PACK];
        from[ph][r] = BF ? -kMid * y.x : 0.f;
        all[ph][r] = y.y;
      }

    f32x4 acc[NA];
#pragma unroll
    for (int i = 0; i < NA; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m[RV], l[RV], mids[NPH];
#pragma unroll
    for (int v = 0; v < RV; ++v) m[v] = -INFINITY, l[v] = 0.f;
    f32x4 offs[NPH];  // (bf16) kMid times the sum of the factors, in every element
#pragma unroll
    for (int ph = 0; ph < NPH; ++ph) {
      mids[ph] = 0.f;
      offs[ph] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    bf16x8 mid8;
#pragma unroll
    for (int e = 0; e < 8; ++e) mid8[e] = (__bf16)kMid;

    auto& st = sh.w[wave];
    for (; key0 < k_hi; key0 += STEP) {
      // ---- what has arrived goes through the LDS (a piece's place goes by its token: the 16 rows that are read together
      // fall on all banks)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.v[16 * i + lane / 4][lane % 4 ^ (QD == 4 ? lane / 16 : lane / 32)] = vq[i];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint32_t kp = there ? kpq[g] : 0u, vp = there ? vpq[g] : 0u;  // (what stands in slots that no row sees may be anything)
        st.ks[lane][g] = __uint_as_float(kp << 16);
        st.km[lane][g] = __uint_as_float(kp & 0xffff0000u);
        st.vs[j][g][n] = __uint_as_float(vp << 16);
        st.vm[j][g][n] = __uint_as_float(vp & 0xffff0000u);
      }
      const uint64_t exist = __ballot(there);
      const bool full = exist == ~0ull && key0 + kKeys - 1 <= least;  // all rows see all keys
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_sched_barrier(0);
      const Pages pg = pn;
      load_v(pg, key0 + STEP);  // (V's registers take the next tile's codes, which the LDS has now)
      pn = pages(key0 + 2 * STEP);
      __builtin_amdgcn_sched_barrier(0);

      // ---- S: s[i][v] is key key0 + 16 i + n of row RV j + v
      float s[4][RV];
      uint32_t kc[4][QD];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int f = 0; f < QD; ++f) kc[i][f] = kq[i][f];
        if constexpr (ALIGNED) by_channels(kc[i]);
      }
#pragma unroll
      for (int ph = 0; ph < NPH; ++ph) {
        uint32_t own = quad_group == ph * PACK + gp ? ~0u : 0u;
        int at = lane;
        if constexpr (!HELD) asm volatile("" : "+v"(own), "+v"(at));  // (read and masked here each time: kept for all phases, Q would spill)
        f32x4 y[4], all_ph;
        if constexpr (SUMS_HELD) {
          all_ph = all[ph];
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = from[ph];
        } else {
          int at_row = RV * j;
          asm volatile("" : "+v"(at_row));  // (read here each time)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float2 q2 = sh.sum[at_row + r / PACK][ph * PACK + r % PACK];
            all_ph[r] = q2.y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i][r] = BF ? -kMid * q2.x : 0.f;
          }
        }
#pragma unroll
        for (int f = ALIGNED ? ph * (QD / NG) : 0; f < (ALIGNED ? (ph + 1) * (QD / NG) : QD); ++f) {
          bf16x8 k8[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) k8[i] = open(kc[i][f]);
#pragma unroll
          for (int part = QP - 1; part >= 0; --part) {
            u32x4 qq;
            if constexpr (HELD) qq = q[part][f];
            else qq = sh.q[part][f][at];
            if constexpr (NPH > 1 && !ALIGNED)
#pragma unroll
              for (int z = 0; z < 4; ++z) qq[z] &= own;
            // (four sums side by side: a product waits for the one before it in its sum)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              y[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qq), k8[i], y[i], 0, 0, 0);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float ks[PACK], km[PACK];
#pragma unroll
          for (int g = 0; g < PACK; ++g) ks[g] = st.ks[16 * i + n][ph * PACK + g], km[g] = st.km[16 * i + n][ph * PACK + g];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float& x = s[i][r / PACK];
            const float z = km[r % PACK] * all_ph[r];
            x = fmaf(ks[r % PACK], y[i][r], ph == 0 && r % PACK == 0 ? z : x + z);
          }
        }
      }
      load_k(pg);  // (K's registers take the next tile's codes as soon as the scores are formed)
      __builtin_amdgcn_sched_barrier(0);

      // ---- running maximum and sum; s becomes P
      if (!full) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int v = 0; v < RV; ++v)
            s[i][v] = (exist >> (16 * i + n) & 1) && key0 + 16 * i + n <= sees[v] ? s[i][v] : -INFINITY;
      }
      float mx[RV];
      bool more = false;
#pragma unroll
      for (int v = 0; v < RV; ++v) {
        mx[v] = row_max(fmaxf(fmaxf(s[0][v], s[1][v]), fmaxf(s[2][v], s[3][v])));
        more |= mx[v] > m[v];
      }
      if (__ballot(more) != 0) {
#pragma unroll
        for (int v = 0; v < RV; ++v) {
          const float m_new = fmaxf(m[v], mx[v]);
          const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[v] - m_new) * c);
          m[v] = m_new;
          l[v] *= alpha;
          if (n == 0) st.alpha[RV * j + v] = alpha;
        }
        __builtin_amdgcn_wave_barrier();
        const float alpha = st.alpha[row];
#pragma unroll
        for (int ph = 0; ph < NPH; ++ph) {
          mids[ph] *= alpha;
          if constexpr (RUNS) offs[ph] *= alpha;
        }
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int f = 0; f < 4; ++f) acc[i][f] *= alpha;
      }
#pragma unroll
      for (int v = 0; v < RV; ++v) {
        // (the difference first: the largest score's weight is 1 exactly, however large it is)
        const float m0 = m[v] == -INFINITY ? 0.f : m[v];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f((s[i][v] - m0) * c);
          l[v] += p;
          st.p[RV * j + v][16 * i + n] = p;
        }
      }
      __builtin_amdgcn_wave_barrier();

      // ---- O^T, a phase's groups at a time: element e is key key0 + 16 j + e of the lane's column
      f32x4 pe[4];
#pragma unroll
      for (int f = 0; f < 4; ++f) pe[f] = *(const f32x4*)&st.p[row][16 * j + 4 * f];
      const uint32_t seen = (uint32_t)(exist >> 16 * j) & ((1u << min(max(last + 1 - (key0 + 16 * j), 0), 16)) - 1u);
#pragma unroll
      for (int ph = 0; ph < NPH; ++ph) {
        float p[16], mid[16];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const f32x4 vs = *(const f32x4*)&st.vs[j][ph * PACK + gp][4 * f], vm = *(const f32x4*)&st.vm[j][ph * PACK + gp][4 * f];
#pragma unroll
          for (int r = 0; r < 4; ++r) p[4 * f + r] = vs[r], mid[4 * f + r] = vm[r];
        }
        if (!full) {  // (a value that the column does not see must not reach it even as 0 times what it holds)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            p[e] = seen >> e & 1 ? p[e] : 0.f;
            mid[e] = seen >> e & 1 ? mid[e] : 0.f;
          }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          mids[ph] = fmaf(pe[e / 4][e % 4], mid[e], mids[ph]);
          p[e] = pe[e / 4][e % 4] * (e & 4 ? -p[e] : p[e]);
        }
        bf16x8 pt[2][PP];
#pragma unroll
        for (int f = 0; f < 2; ++f) {  // (in open8's order)
          const float x8[8] = {p[8 * f], p[8 * f + 4], p[8 * f + 1], p[8 * f + 5], p[8 * f + 2], p[8 * f + 6], p[8 * f + 3], p[8 * f + 7]};
          split<PP>(x8, pt[f]);
        }
        if constexpr (RUNS)
#pragma unroll
        for (int part = PP - 1; part >= 0; --part)
#pragma unroll
          for (int f = 0; f < 2; ++f) offs[ph] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mid8, pt[f][part], offs[ph], 0, 0, 0);
#pragma unroll
        for (int i = ph * PACK * (NA / NG); i < (ph + 1) * PACK * (NA / NG); i += SIDE) {
          bf16x8 v8[SIDE][2];
          f32x4 z[SIDE];
#pragma unroll
          for (int y = 0; y < SIDE; ++y) {
            // 16 keys of channel 16 (i + y) + n: the lane's row of the LDS is key 16 j + n
            const int piece = QD == 4 ? (i + y) / 2 ^ n / 4 : (i + y) ^ n / 8;
            const char* row_at = (const char*)&st.v[16 * j + n][piece] + (QD == 4 ? (i + y) % 2 * 8 : 0);
            const i32x2 v = __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) i32x2*)row_at);
            v8[y][0] = open((uint32_t)v[0]);
            v8[y][1] = open((uint32_t)v[1]);
            z[y] = RUNS ? acc[i + y] : f32x4{0.f, 0.f, 0.f, 0.f};
          }
#pragma unroll
          for (int part = PP - 1; part >= 0; --part)
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
              for (int y = 0; y < SIDE; ++y) z[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8[y][f], pt[f][part], z[y], 0, 0, 0);
#pragma unroll
          for (int y = 0; y < SIDE; ++y) acc[i + y] = RUNS ? z[y] : acc[i + y] + z[y];
        }
      }
      __builtin_amdgcn_wave_barrier();  // the tile's LDS is read
    }

    // ---- the next run, its first tile in flight under this one's end
    const int cur_b = b, cur_item = item, cur_h = h;
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
#pragma unroll
    for (int v = 0; v < RV; ++v) l[v] = row_sum(l[v]);
#pragma unroll
    for (int ph = 0; ph < NPH; ++ph) mids[ph] = column_sum(mids[ph]);
    __syncthreads();  // sh.q and the tiles are read
    if (n == 0)
#pragma unroll
      for (int v = 0; v < RV; ++v) {
        sM[wave][RV * j + v] = m[v];
        sL[wave][RV * j + v] = l[v];
      }
    if (row < nrows)
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const int g = i / (NA / NG);
        if (g % PACK != gp) continue;
#pragma unroll
        for (int f = 0; f < 4; ++f) sh.o[wave][row][16 * i + 4 * j + f] =
              fmaf(16.f, RUNS ? acc[i][f] - offs[g / PACK][f] : acc[i][f], mids[g / PACK]);
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
      T* out = (T*)ka.a.o + cur_b * ka.a.osb + hq * ka.a.osh + tk * ka.a.oss + d;
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const float y = none ? 0.f : o[f] * inv;
        if constexpr (BF) ((__bf16*)out)[f] = (__bf16)y;
        else out[f] = y;
      }
      if (ka.a.lse != nullptr && d == 0)
        ka.a.lse[((int64_t)cur_b * a.heads_q + hq) * a.tokens + tk] =
            none ? -INFINITY : ((mx == -INFINITY ? 0.f : mx * c) + __log2f(sum)) * kLn2;
    }
    if (ka.join && opens && tid == 0)
      ka.record[(int64_t)cur_b * items + cur_item] = whole ? make_int2(-1, -1) : make_int2(slot, deal.owner(row_last));
    if (!busy) break;
    first_run = false;
    __syncthreads();  // sh.o is read
  }
}

// Groups that share the columns: as many as the rows leave room for, since each phase opens and weighs the tile again (8 x 8192 tokens in groups
// of 32: 8 rows of each of 8 heads, two phases, 36 us; 16 rows of each of 4, four phases, half the tiles, 37).
int pack_of(int groups, int rows) {
  int pack = groups;
  while (pack > 1 && rows > 16 / pack) pack /= 2;
  return pack;
}

struct Plan {
  int group, rows, groups, pack, block, row_blocks;
  size_t ml, o, total;  // byte offsets in the workspace (the records come first)
};
Plan plan(int batch, int heads_q, int heads_kv, int tokens, int head_dim, int elements) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  Plan p;
  p.group = heads_q / heads_kv;
  p.rows = p.group * tokens;
  p.groups = head_dim / elements;
  p.pack = pack_of(p.groups, p.rows);
  p.block = 16 / p.pack;
  p.row_blocks = (p.rows + p.block - 1) / p.block;
  p.ml = up((size_t)batch * heads_kv * p.row_blocks * sizeof(int2));
  p.o = p.ml + up((size_t)2 * kWorkers * p.block * sizeof(float2));
  p.total = p.o + (size_t)2 * kWorkers * p.block * head_dim * sizeof(float);
  return p;
}

template <typename T, int D, int NG, int PACK, int QP>
hipError_t launch(const KernelArgs& k, dim3 grid, hipStream_t s) {
  // (key by key costs registers: 28 rotated rows spill 105 of them instead of 61)
  const int64_t far = (int64_t)1 << 26;  // (16 rows of a run within 2^30 bytes)
  const CacheArgs& ca = k.a.q.cache;
  if (ca.table.page.d % 16 == 0 && ca.k.ss < far && ca.v.ss < far) q4_attn_kernel<T, D, NG, PACK, QP, true><<<grid, kThreads, 0, s>>>(k);
  else q4_attn_kernel<T, D, NG, PACK, QP, false><<<grid, kThreads, 0, s>>>(k);
  return hipGetLastError();
}
template <typename T, int D, int NG, int PACK>
hipError_t launch(const KernelArgs& k, dim3 grid, hipStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (!k.a.q.rope.freq) return launch<T, D, NG, PACK, 1>(k, grid, s);
  return launch<T, D, NG, PACK, 3>(k, grid, s);
}
template <typename T, int D, int NG>
hipError_t launch(const KernelArgs& k, const Plan& p, dim3 grid, hipStream_t s) {
  hipError_t e = hipErrorInvalidValue;
  if (p.pack == 1) e = launch<T, D, NG, 1>(k, grid, s);
  if constexpr (NG >= 2)
    if (p.pack == 2) e = launch<T, D, NG, 2>(k, grid, s);
  if constexpr (NG >= 4)
    if (p.pack == 4) e = launch<T, D, NG, 4>(k, grid, s);
  if (e != hipSuccess || !k.join) return e;
  const QueryArgs& a = k.a.q;
  return launch_join<T, D>({k.record, k.part_ml, k.part_o, k.a.o, k.a.osb, k.a.osh, k.a.oss, k.a.lse, k.group, k.blocks, a.batch,
                            a.heads_q, a.cache.heads_kv, a.tokens, k.rows, k.row_blocks, p.block, k.scale_log2}, s);
}
template <typename T>
hipError_t launch(const KernelArgs& k, const Plan& p, dim3 grid, hipStream_t s) {
  if (k.a.q.cache.head_dim == 128)
    return p.groups == 4 ? launch<T, 128, 4>(k, p, grid, s) : launch<T, 128, 2>(k, p, grid, s);
  return p.groups == 2 ? launch<T, 64, 2>(k, p, grid, s) : launch<T, 64, 1>(k, p, grid, s);
}

}  // namespace

size_t q4_attn_workspace(int batch, int heads_q, int heads_kv, int tokens, int head_dim, int group) {
  return plan(batch, heads_q, heads_kv, tokens, head_dim, group).total;
}

hipError_t launch_q4_attn(const Q4AttnArgs& a, hipStream_t s) {
  const QueryArgs& q = a.q;
  const Plan p = plan(q.batch, q.heads_q, q.cache.heads_kv, q.tokens, q.cache.head_dim, q.cache.group);
  KernelArgs k;
  k.a = a;
  auto strides = [&](const PoolView& v) -> PoolStrides {
    return {(uint32_t)(v.sp / 16), (uint32_t)(v.ss / 16), (uint32_t)(v.psp / p.groups), (uint32_t)(v.pss / p.groups)};
  };
  k.kst = strides(q.cache.k);
  k.vst = strides(q.cache.v);
  k.group = fast_div(p.group);
  k.blocks = fast_div(p.row_blocks);
  k.rows = p.rows;
  k.row_blocks = p.row_blocks;
  k.capacity = q.cache.table.max_pages * q.cache.table.page.d;  // (at most 2^30: no sum of keys overflows)
  const int64_t rows = (int64_t)q.batch * q.cache.heads_kv * p.row_blocks;  // a KV head's, as the workgroups take them
  k.join = k.capacity > kWholeKeys;
  // a unit is a tile for each wavefront; a whole row where rows are not split, and more where the weights of all units
  // would not stay below 2^30
  k.unit_shift = 8;
  static_assert(kWaves * kKeys == 1 << 8, "keys of a unit");
  auto units = [&]() -> int64_t { return ((int64_t)k.capacity + ((int64_t)1 << k.unit_shift) - 1) >> k.unit_shift; };
  while ((!k.join && units() > 1) || (units() + 2) * rows > (1 << 30)) ++k.unit_shift;
  k.scale_log2 = 16.f * q.scale * kLog2e;
  char* ws = (char*)a.workspace;
  k.record = (int2*)ws;
  k.part_ml = (float2*)(ws + p.ml);
  k.part_o = (float*)(ws + p.o);
  const dim3 grid((unsigned)std::min((int64_t)kWorkers, units() * rows));
  return q.bf16 ? launch<uint16_t>(k, p, grid, s) : launch<float>(k, p, grid, s);
}

}  // namespace seer
