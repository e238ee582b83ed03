// q4_attn_kernels.hip -- attention of new tokens over a paged cache held in 4 bits.
//
// As over a cache of values (paged_attn_kernels.hip) the rows of a KV group are the columns of S^T = K Q^T and O^T = V^T P^T, and
// the units of all sequences' keys are dealt out evenly to the workgroups.  What differs is that a key is 40 to 80 bytes and
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
// sign, the second product's sums would be 5 to 100 times the result and carry their rounding into it.)
//
// Columns.  A step belongs to a group, so that a group's products may not run into another's sum.  Where a block has
// few rows (16 / (D / group) at most), its columns are pairs of row and group: the operand Q^T is 0 but in the
// column's group, which gives S^T by groups in one accumulator, and P^T in column (g, r) is p step_g, of which the
// outputs of group g take theirs: no weight is formed twice, and the lanes of a row add up its score by two exchanges.  With
// more rows the columns are rows alone (or of two groups), and the groups are done one after the other.
//
// A wavefront takes 64 keys at a time.  K's codes come to registers as the operand wants them (16 bytes of one
// key a lane); V's go through the wavefront's own LDS and come back transposed (ds_read_b64_tr_b4: 16 keys of
// one channel a lane); so do both params, from a token a lane to the 16 keys of a lane's scores.
//
// Precision: fp32 statistics and sums; p step enters the second product in three bf16 parts, which hold fp32 whole, and
// so does a q that is rotated here or fp32 the first.
#include <algorithm>

#include "cache.h"
#include "paged_join.h"
#include "q4_open.h"

namespace seer {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kKeys = 64;      // of a tile
constexpr int kWholeKeys = 512;  // rows with room for so many are not split

struct KernelArgs {
  Q4AttnArgs a;
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

// x[0 .. 7] as three bf16 parts in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ void split3_order(const float (&x)[8], bf16x8 (&y)[3]) {
  const float z[8] = {x[0], x[4], x[1], x[5], x[2], x[6], x[3], x[7]};
  split3(z, y);
}

typedef __attribute__((ext_vector_type(2))) int i32x2;

// D: elements of a head.  NG: groups of a head.  PACK: of them, those that share the columns.  QP: bf16 parts of q.
// RUN: pages hold whole aligned runs of 16 keys.
template <typename T, int D, int NG, int PACK, int QP, bool RUN>
__global__ __launch_bounds__(kThreads, 2) void q4_attn_kernel(KernelArgs ka) {
  constexpr int ROWS = 16 / PACK, NPH = NG / PACK;
  constexpr int NA = D / 16;           // accumulators: 16 channels each
  constexpr int QD = D / 32;           // dwords of a key's codes per lane; 16-byte pieces of a V row
  constexpr int NI = QD;               // loads of V's codes per lane
  constexpr int TQ = 16 / QD;          // tokens of a run that one of them brings
  constexpr int OSTR = D + 4;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int kRowCost = 1;          // a row's beginning and end, in units
  constexpr int PIECES = D / 8;
  __shared__ union {
    struct {
      u32x4 q[QP][ROWS][PIECES];       // 8 elements in open8's order, 4 to 7 negated
      float2 sum[ROWS][NG];            // of a row's elements in a group: as above, and all / 16
      float2 cs[ROWS][D / 2];
      struct {
        u32x4 v[NI][kWave];
        uint32_t kp[4][NG][16], vp[4][NG][16];  // params by run, group, key
      } w[kWaves];
    };
    float o[kWaves][ROWS][OSTR];
  } sh;
  __shared__ float sM[kWaves][ROWS], sL[kWaves][ROWS];

  const QueryArgs& a = ka.a.q;
  const CacheArgs& ca = a.cache;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane % 16, j = lane / 16;  // column, run of 16 keys
  const int gp = n / ROWS, row = n % ROWS;
  const int items = ca.heads_kv * ka.row_blocks;  // rows of a sequence
  const int group = ka.group.d;
  const float c = ka.scale_log2;
  const bool rope = (QP == 3 || !BF) && a.rope.freq != nullptr;
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

  // ---- a run of one row's units [u0, u1)
  int u0, u1, h, key0, k_hi;
  const char *kbase, *vbase;
  const uint32_t *kpbase, *vpbase;
  const int32_t* table;

  // K: lane row n of sub-tile i is key 16 (n / 4) + 4 i + n % 4; V's codes: load i brings token 16 j + i TQ + n / QD;
  // params: token `lane`.
  const int kk = n / 4 * 16 + n % 4, vk = 16 * j + n / QD;
  struct Pages {
    int k[RUN ? 1 : 4], v[RUN ? 1 : NI], p;
  };
  // (A key past the run is looked up at the run's last one and then has no page.)
  auto page_of = [&](int key) -> int {
    const int page = table[fast_quot(ca.table.page, max(min(key, k_hi - 1), 0))];
    return key < k_hi ? page : -1;
  };
  auto pages = [&](int key0) -> Pages {
    Pages p;
    if constexpr (RUN) {
      p.k[0] = page_of(key0 + n / 4 * 16);  // (the run's first key: it exists where any of them does)
      p.v[0] = page_of(key0 + 16 * j);
      p.p = p.v[0];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) p.k[i] = page_of(key0 + kk + 4 * i);
#pragma unroll
      for (int i = 0; i < NI; ++i) p.v[i] = page_of(key0 + vk + i * TQ);
      p.p = page_of(key0 + lane);
    }
    return p;
  };
  // Page and slot of a key (the pool's first slot where its page is none).
  struct At {
    int page, slot;
  };
  auto place = [&](int page, int key) -> At {
    const bool ok = (uint32_t)page < (uint32_t)ca.table.num_pages;
    const int slot = key - fast_quot(ca.table.page, key) * ca.table.page.d;
    return {ok ? page : 0, ok ? slot : 0};
  };

  uint32_t kq[4][QD];     // K's codes: 8 QD elements of key 16 (n / 4) + 4 i + n % 4
  u32x4 vq[NI];           // V's, on their way
  uint32_t kpq[NG], vpq[NG];
  bool there;             // token `lane` exists
  auto load_k = [&](const Pages& pg, int key0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = key0 + kk + 4 * i;
      At s = place(pg.k[RUN ? 0 : i], RUN ? key0 + kk : key);
      if (RUN) s.slot += 4 * i;
      const char* p = kbase + s.page * ca.k.sp + s.slot * ca.k.ss;
      if constexpr (QD == 4) {
        const u32x4 z = *(const u32x4*)p;
#pragma unroll
        for (int f = 0; f < 4; ++f) kq[i][f] = z[f];
      } else {
        const u32x2 z = *(const u32x2*)p;
        kq[i][0] = z[0];
        kq[i][1] = z[1];
      }
    }
  };
  auto load_v = [&](const Pages& pg, int key0) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int key = key0 + vk + i * TQ;
      At s = place(pg.v[RUN ? 0 : i], RUN ? key0 + vk : key);
      if (RUN) s.slot += i * TQ;
      // (a piece's place in the LDS goes by the load: the 16 rows that are read together fall on all banks)
      vq[i] = *(const u32x4*)(vbase + s.page * ca.v.sp + s.slot * ca.v.ss + 16 * ((n ^ i) % QD));
    }
    const int key = key0 + lane;
    const At s = place(pg.p, key);
    there = (uint32_t)pg.p < (uint32_t)ca.table.num_pages && key < k_hi;
    const uint32_t* kp = kpbase + s.page * ca.k.psp + s.slot * ca.k.pss;
    const uint32_t* vp = vpbase + s.page * ca.v.psp + s.slot * ca.v.pss;
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
    kbase = (const char*)ca.k.data + h * ca.k.sh + 4 * QD * j;
    vbase = (const char*)ca.v.data + h * ca.v.sh;
    kpbase = ca.k.params + h * ca.k.psh;
    vpbase = ca.v.params + h * ca.v.psh;
    table = ca.table.ptr + b * ca.table.stride;
    const Pages pg = pages(key0);
    pn = pages(key0 + STEP);
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
      const int32_t* rpos_b = a.rope_positions + b * a.pos_stride;
      if (lane < a.rope.rot / 2) {
        for (int tk = t_first + wave; tk <= t_last; tk += kWaves) {
          float co, si;
          turn_cos_sin(rate, rpos_b[tk], co, si);
          sh.cs[tk - t_first][lane] = make_float2(co * a.rope.scale, si * a.rope.scale);
        }
      }
      __syncthreads();
    }
    static_assert(ROWS * PIECES <= kThreads, "one piece a thread");
    if (tid < ROWS * PIECES) {
      const int rl = tid / PIECES, d0 = tid % PIECES * 8;
      const int r = min(r0 + rl, ka.rows - 1), tk = fast_quot(ka.group, r);
      const T* src = (const T*)a.q.ptr + b * a.q.sb + (h * group + (r - tk * group)) * a.q.sh + tk * a.q.ss;
      const bool turns = rope && d0 < a.rope.rot;
      float y[8], z[8];
      u32x4 raw[BF ? 1 : 2];
#pragma unroll
      for (int f = 0; f < (BF ? 1 : 2); ++f) raw[f] = *((const u32x4*)(src + d0) + f);
      unpack8(raw, y);
      if (turns) {
        const int half = a.rope.rot / 2;
        const T* other = src + (a.rope.interleaved ? d0 : d0 < half ? d0 + half : d0 - half);
#pragma unroll
        for (int f = 0; f < (BF ? 1 : 2); ++f) raw[f] = *((const u32x4*)other + f);
        unpack8(raw, z);
        rotate8(a.rope, sh.cs[tk - t_first], d0, y, z);
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
      if constexpr (QP == 3) {
        bf16x8 z3[3];
        split3(s8, z3);
#pragma unroll
        for (int part = 0; part < 3; ++part) sh.q[part][rl][tid % PIECES] = __builtin_bit_cast(u32x4, z3[part]);
      } else {
        u32x4 z1;
#pragma unroll
        for (int f = 0; f < 4; ++f)
          z1[f] = __builtin_amdgcn_perm(__float_as_uint(s8[2 * f + 1]), __float_as_uint(s8[2 * f]), 0x07060302u);
        sh.q[0][rl][tid % PIECES] = z1;
      }
    }
    // the last key that the lane's column sees (none beyond the rows)
    const int my_row = min(r0 + row, ka.rows - 1);
    const int last = min(pos_b[fast_quot(ka.group, my_row)], ka.capacity - 1);
    __syncthreads();

    // the operand Q^T, 0 but in the column's group (where the columns hold all of them)
    const int quad_group = j * NG / 4;
    u32x4 q[QP][QD];
    float2 qsum[NPH];
#pragma unroll
    for (int part = 0; part < QP; ++part)
#pragma unroll
      for (int i = 0; i < QD; ++i) {
        q[part][i] = sh.q[part][row][j * QD + i];
        if constexpr (NPH == 1)
#pragma unroll
          for (int f = 0; f < 4; ++f) q[part][i][f] = quad_group == gp ? q[part][i][f] : 0u;
      }
#pragma unroll
    for (int ph = 0; ph < NPH; ++ph) qsum[ph] = sh.sum[row][ph * PACK + gp];

    f32x4 acc[NA];
#pragma unroll
    for (int i = 0; i < NA; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f, mids[NPH];
#pragma unroll
    for (int ph = 0; ph < NPH; ++ph) mids[ph] = 0.f;

    auto& st = sh.w[wave];
    for (; key0 < k_hi; key0 += STEP) {
      // ---- what has arrived goes through the LDS
#pragma unroll
      for (int i = 0; i < NI; ++i) st.v[i][lane] = vq[i];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        st.kp[j][g][n] = there ? kpq[g] : 0u;  // (what stands in slots that no row sees may be anything)
        st.vp[j][g][n] = there ? vpq[g] : 0u;
      }
      const uint32_t exist = (uint32_t)(__ballot(there) >> 16 * j) & 0xffffu;
      __builtin_amdgcn_wave_barrier();

      // ---- S^T: element e is key key0 + 16 j + e of the lane's column
      float s[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int ph = 0; ph < NPH; ++ph) {
        const uint32_t own = quad_group == ph * PACK + gp ? ~0u : 0u;
        u32x4 kp[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) kp[f] = *(const u32x4*)&st.kp[j][ph * PACK + gp][4 * f];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y0 = -kMid * qsum[ph].x;
          f32x4 y = {y0, y0, y0, y0};
#pragma unroll
          for (int part = QP - 1; part >= 0; --part)
#pragma unroll
            for (int f = 0; f < QD; ++f) {
              u32x4 qq = q[part][f];
              if constexpr (NPH > 1)
#pragma unroll
                for (int z = 0; z < 4; ++z) qq[z] &= own;
              y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(open8(kq[i][f]), __builtin_bit_cast(bf16x8, qq), y, 0, 0, 0);
            }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t p = kp[i][r];
            s[4 * i + r] = fmaf(__uint_as_float(p << 16), y[r], fmaf(__uint_as_float(p & 0xffff0000u), qsum[ph].y, s[4 * i + r]));
          }
        }
      }
      if constexpr (PACK >= 2)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = dpp_add<0x128>(s[e]);  // row_ror 8
      if constexpr (PACK == 4)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = dpp_add<0x124>(s[e]);  // row_ror 4

      const Pages pg = pn;
      pn = pages(key0 + 2 * STEP);
      load_k(pg, key0 + STEP);
      load_v(pg, key0 + STEP);

      // ---- running maximum and sum; s becomes P
      const uint32_t seen = exist & ((1u << min(max(last + 1 - (key0 + 16 * j), 0), 16)) - 1u);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = seen >> e & 1 ? s[e] : -INFINITY;
      float mx = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
      mx = column_max(mx);
      if (__ballot(mx > m) != 0) {
        const float m_new = fmaxf(m, mx);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - m_new) * c);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int ph = 0; ph < NPH; ++ph) mids[ph] *= alpha;
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int f = 0; f < 4; ++f) acc[i][f] *= alpha;
      }
      // (the difference first: the largest score's weight is 1 exactly, however large it is)
      const float m0 = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = __builtin_amdgcn_exp2f((s[e] - m0) * c);
        l += s[e];
      }

      // ---- O^T, a phase's groups at a time
      const bool partly = __ballot(seen != exist) != 0;
#pragma unroll
      for (int ph = 0; ph < NPH; ++ph) {
        float p[16], mid[16];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const u32x4 vp = *(const u32x4*)&st.vp[j][ph * PACK + gp][4 * f];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            p[4 * f + r] = __uint_as_float(vp[r] << 16);
            mid[4 * f + r] = __uint_as_float(vp[r] & 0xffff0000u);
          }
        }
        if (partly) {  // (a value that the column does not see must not reach it even as 0 times what it holds)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            p[e] = seen >> e & 1 ? p[e] : 0.f;
            mid[e] = seen >> e & 1 ? mid[e] : 0.f;
          }
        }
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          mids[ph] = fmaf(s[e], mid[e], mids[ph]);
          p[e] *= e & 4 ? -s[e] : s[e];
          sum += p[e];
        }
        const float z0 = -kMid * column_sum(sum);
        bf16x8 pt[2][3];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const float x8[8] = {p[8 * f], p[8 * f + 1], p[8 * f + 2], p[8 * f + 3], p[8 * f + 4], p[8 * f + 5], p[8 * f + 6], p[8 * f + 7]};
          split3_order(x8, pt[f]);
        }
#pragma unroll
        for (int i = ph * PACK * (NA / NG); i < (ph + 1) * PACK * (NA / NG); ++i) {
          // 16 keys of channel 16 i + n: the lane's row of the LDS is key 16 j + n
          const int li = n / TQ;  // the load that brought it
          const char* row_at = (const char*)&st.v[li][16 * j + n % TQ * QD + ((i / 2) ^ li) % QD] + i % 2 * 8;
          const i32x2 v = __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) i32x2*)row_at);
          f32x4 z = {z0, z0, z0, z0};
#pragma unroll
          for (int part = 2; part >= 0; --part)
#pragma unroll
            for (int f = 0; f < 2; ++f)
              z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(open8((uint32_t)v[f]), pt[f][part], z, 0, 0, 0);
          acc[i] += z;
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
    l = column_sum(l);
#pragma unroll
    for (int ph = 0; ph < NPH; ++ph) mids[ph] = column_sum(mids[ph]);
    __syncthreads();  // sh.q and the tiles are read
    if (gp == 0 && j == 0) {
      sM[wave][row] = m;
      sL[wave][row] = l;
    }
    if (row < nrows)
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const int g = i / (NA / NG);
        if (g % PACK != gp) continue;
#pragma unroll
        for (int f = 0; f < 4; ++f) sh.o[wave][row][16 * i + 4 * j + f] = fmaf(16.f, acc[i][f], mids[g / PACK]);
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

// Columns that are shared by groups, rows of a block.
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
  if (k.a.q.cache.table.page.d % 16 == 0) q4_attn_kernel<T, D, NG, PACK, QP, true><<<grid, kThreads, 0, s>>>(k);
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
