// weights_kernels.hip -- the attention weight that each cached key gets from some queries (seer_kv_weights).
//
//   out[t] = decay in[t] + sum over the rows r that see t of exp(scale q_r . k_t - lse_r)
//
// The half of attention that needs no running maximum: the rows' log-sum-exps are known, so that a key's sum is
// its own affair.  A wavefront holds 64 keys (32 of fp32) as one operand of S = Q K^T and goes through the rows, 16
// rows of the other operand at a time; a lane adds up its keys' weights over its rows, and the quads of lanes, which hold different
// rows of the same keys, are joined at the end.  So the keys are read once however many rows there are, a key belongs to one
// wavefront, and there are no atomics.
//
// Units of keys are dealt out to the workgroups as in attention, and keys in 4 bits enter as there
// (q4_attn_kernels.hip), centred for a q in fp32 (a rotated row over 70 and 300 keys: weights 0.8e-7 to 2.5e-7 off in the 2-norm, and 3e-7 to
// 1.0e-6 with codes of one sign, 0.7e-6 to 3.3e-6 where one element of each group is far off; 131072 tokens of 32 / 8 heads of 128 30 us, and 25).  A
// head's rows stay in the LDS for all units of a run, where they fit.
//
// Measured (bf16, 32 / 8 heads of 128, one MI355X): 64 sequences of 200 to 16000 tokens in 4 bits, a token each, 49 us for 170 MB
// (3.4e12 bytes a second; a kernel that only reads reaches 6.2e12), bound by the latency of a tile's loads and a run's beginning;
// the last 64 tokens of 32768 over bf16 keys, 43 us for 68 MB: 256 rows, whose exponentials, products and sums take half of the
// units' time; the rest is waits for the rows' operands and factors out of the LDS.
#include <algorithm>

#include "cache.h"
#include "q4_open.h"

namespace seer {

namespace {

constexpr int kRoom = 72 << 10;  // bytes of LDS for rows: two workgroups of a CU hold the rows of 64 tokens of 4 heads of 128 each

struct KernelArgs {
  WeightArgs a;
  int64_t ksp, ksh, kss;  // K's strides in bytes
  int rows;               // G tokens
  int blocks, held;       // blocks of rows, and those that the LDS holds at a time
  FastDiv group;
  int capacity;           // keys that are counted at most
  int unit_shift;         // log2 of the keys per unit
  float scale;            // of a score (4 bits: of a score / 16)
};

// Keys of a sequence that are counted: those up to its tokens' last position.
__device__ __forceinline__ int length_of(const KernelArgs& k, int b) {
  int len = 0;
  const int32_t* p = k.a.q.positions + b * k.a.q.pos_stride;
  for (int s = 0; s < k.a.q.tokens; ++s) len = max(len, min(p[s], k.capacity - 1) + 1);
  return len;
}
__device__ __forceinline__ int units_of(const KernelArgs& k, int len) {
  return (len + (1 << k.unit_shift) - 1) >> k.unit_shift;
}

// T: type of q, and of the keys where NG is 0 (else: 4 bits, NG groups of a head, PACK of them sharing the operand's rows).
// QP: bf16 parts of q (1: bf16 as it is, or fp32 keys; 3, which hold fp32 whole: rotated, or fp32 over 4 bits).
template <typename T, int D, int NG, int PACK, int QP>
struct Shape {
  static constexpr bool BF = sizeof(T) == 2, Q4 = NG != 0, F32 = !BF && !Q4;
  static constexpr int SUB = F32 ? 2 : 4;              // sub-tiles of 16 keys
  static constexpr int KT = 16 * SUB;
  static constexpr int ROWS = 16 / PACK;               // rows of a block
  static constexpr int STEPS = F32 ? D / 16 : D / 32;  // 16-byte pieces of Q per lane
  static constexpr int NGX = Q4 ? NG : 1;
  static constexpr bool TURNS = QP > 1 || F32;         // q may be rotated here
  struct Row {                                         // of a row in the LDS
    float lse;
    int last;                                          // the last key that it sees
    float2 sum[NGX];                                   // as in q4_attn_kernel
  };
  // of a block: the operand as the lanes read it, rows, cosines and sines of their tokens
  static constexpr int OPERAND = QP * STEPS * kWave * 16;
  static constexpr int BYTES = OPERAND + ROWS * (int)sizeof(Row) + (TURNS ? ROWS * (D / 2) * 8 : 0);
  static constexpr int MOST = kRoom > BYTES ? kRoom / BYTES : 1;  // blocks that the LDS holds
  // per SIMD, as the registers allow (4 bits of 128 elements with q in three parts: 4 spill 26, and a token after 131072 takes 39.5
  // us for 27.1)
  static constexpr int WAVES = !Q4 || NG == 1 ? 4 : PACK == 1 ? 2 : D == 128 && QP == 3 ? 3 : 4;
  // few rows: small workgroups, whose shares are finer (64 sequences of 200 tokens 12.8 -> 8.2 us); many: large ones, which share them
  static constexpr int THREADS = Q4 && PACK > 1 ? 256 : 512;
  static constexpr int UNIT_SHIFT = (THREADS == 512 ? 3 : 2) + (F32 ? 5 : 6);  // log2 of a tile for each wavefront
};

template <typename T, int D, int NG, int PACK, int QP, bool RUN>
__global__ __launch_bounds__((Shape<T, D, NG, PACK, QP>::THREADS), (Shape<T, D, NG, PACK, QP>::WAVES)) void weights_kernel(KernelArgs ka) {
  using S = Shape<T, D, NG, PACK, QP>;
  constexpr int kThreads = S::THREADS, kWaves = kThreads / kWave;
  constexpr bool BF = S::BF, Q4 = S::Q4, F32 = S::F32;
  constexpr int SUB = S::SUB, KT = S::KT, ROWS = S::ROWS, STEPS = S::STEPS, NGX = S::NGX;
  constexpr int RV = 4 / PACK;                  // rows whose scores a lane holds
  constexpr int NPH = Q4 ? NG / PACK : 1;
  // as in q4_attn_kernels.hip: the channels of one group a step
  constexpr bool ALIGNED = NPH > 1;
  static_assert(!ALIGNED || PACK == 1, "a block's groups all share the rows, or none");
  constexpr int KW = Q4 ? D / 32 : 4 * STEPS;   // dwords of a key per lane
  auto open = [](uint32_t codes) {
    if constexpr (BF) return open8(codes);
    else return open8_centred(codes);
  };
  extern __shared__ __attribute__((aligned(16))) char room[];
  __shared__ __attribute__((aligned(16))) float sks[kWaves][Q4 ? KT : 1][NGX], skm[kWaves][Q4 ? KT : 1][NGX];
  u32x4(*sq)[QP][STEPS][kWave] = (u32x4(*)[QP][STEPS][kWave])room;
  typename S::Row* srow = (typename S::Row*)(room + ka.held * S::OPERAND);
  float2(*scs)[D / 2] = (float2(*)[D / 2])(srow + ka.held * ROWS);

  const QueryArgs& a = ka.a.q;
  const CacheArgs& ca = a.cache;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane % 16, j = lane / 16;
  const int items = ca.heads_kv;
  const int group = ka.group.d;
  const float c = ka.scale;
  // exp(c s - lse): the difference first, rounded once, then log2(e), so that the power is as exact for large scores as for small ones (both
  // sides times log2(e) first: around 290, weights 7e-6 off instead of 4e-7, 64 tokens over 4096 keys 1.7e-7 instead of 1.1e-7 in the 2-norm;
  // 64 tokens over 32768 38.9 us and 40.2 this way)
  auto power = [&](float s, float lse) { return __builtin_amdgcn_exp2f(fmaf(s, c, -lse) * kLog2e); };
  const bool rope = S::TURNS && a.rope.freq != nullptr;
  const double freq = (rope ? a.rope.freq : (const double*)ca.k.data)[rope ? min(lane, a.rope.rot / 2 - 1) : 0];

  // ---- this workgroup's share (every wavefront works it out by itself)
  const int share = (a.batch + kWave - 1) / kWave;  // sequences per lane
  const int b_lo = min(lane * share, a.batch), b_hi = min(b_lo + share, a.batch);
  int mine = 0, my_len = 0;
  for (int i = b_lo; i < b_hi; ++i) {
    my_len = length_of(ka, i);
    mine += units_of(ka, my_len);
  }
  const int upto = wave_prefix(mine);
  const TurnRate rate = turn_rate(freq);
  const uint32_t total = (uint32_t)(__builtin_amdgcn_readlane(upto, kWave - 1) * items);
  if (blockIdx.x >= total) return;  // (a unit each at least, or none)
  const Deal deal(total, gridDim.x);
  const int w = share_of(ca.k, a.batch, blockIdx.x, (int)min(gridDim.x, total));
  int x = deal.first(w);
  const int x_end = deal.first(w + 1);
  const int owner_lane = (int)__popcll(__ballot(upto * items <= x));
  int b = owner_lane * share;
  int off = x - (__builtin_amdgcn_readlane(upto, owner_lane) - __builtin_amdgcn_readlane(mine, owner_lane)) * items;
  int len = share == 1 ? __builtin_amdgcn_readlane(my_len, owner_lane) : length_of(ka, b);
  int row_units = units_of(ka, len);
  while (off >= row_units * items) {
    off -= row_units * items;
    len = length_of(ka, ++b);
    row_units = units_of(ka, len);
  }
  len = __builtin_amdgcn_readfirstlane(len);
  row_units = __builtin_amdgcn_readfirstlane(row_units);
  int h = (int)((uint32_t)off / (uint32_t)row_units);
  int u0 = off - h * row_units;  // the next unit of the head

  // Keys' operand: lane n of sub-tile i is key 16 i + n of a tile; params: token `lane`.
  int k_hi, last_page;
  const char* kbase;
  const uint32_t* kpbase;
  const int32_t* table;
  uint32_t kq[SUB][KW];
  uint32_t kpq[NGX];
  bool there;  // key `lane` of the tile is counted and its page exists
  struct At {
    int page, slot;
  };
  struct Pages {
    At k[SUB], p;
  };
  // A key's page, as the table has it, and slot.  (A key past the run is taken to be on its last one's page.)
  auto page_of = [&](int key) -> At {
    const int i = fast_quot(ca.table.page, key);
    return {table[min(i, last_page)], key - i * ca.table.page.d};
  };
  auto has_page = [&](int page) { return (uint32_t)page < (uint32_t)ca.table.num_pages; };
  auto pages = [&](int key0) -> Pages {
    Pages p;
    p.p = page_of(key0 + (RUN ? min(lane, KT - 1) / 16 * 16 : min(lane, KT - 1)));
    if constexpr (!RUN)
#pragma unroll
      for (int i = 0; i < SUB; ++i) p.k[i] = page_of(key0 + 16 * i + n);
    return p;
  };
  const int klane = (RUN ? n * (int)ka.kss : 0) + (Q4 ? 4 * KW : 16) * j;
  // Byte offset of a key's row (the pool's first page where it has none).
  auto offset = [&](const At& s) { return (has_page(s.page) ? s.page : 0) * ka.ksp + s.slot * ka.kss; };
  auto load = [&](const Pages& pg, int key0) {
    // (a lane forms its run's offset, for all: sixteen scalar products a tile were a third of its time)
    const int64_t mine = RUN ? offset(pg.p) : 0;
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
      int64_t off;
      if constexpr (RUN)
        off = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), 16 * i) << 32 |
                        (uint32_t)__builtin_amdgcn_readlane((int)mine, 16 * i));
      else off = offset(pg.k[i]);
      const char* p = kbase + off + (uint32_t)klane;
      if constexpr (KW == 2) {
        const u32x2 z = __builtin_nontemporal_load((const u32x2*)p);
        kq[i][0] = z[0];
        kq[i][1] = z[1];
      } else {
#pragma unroll
        for (int f = 0; f < KW / 4; ++f) {
          // (codes past the caches: 64 mixed sequences 60 -> 51 us; values that way: 64 rows over 32768 tokens 42 -> 44)
          u32x4 z;
          if constexpr (Q4) z = __builtin_nontemporal_load((const u32x4*)(p + 64 * f));
          else z = *(const u32x4*)(p + 64 * f);
#pragma unroll
          for (int y = 0; y < 4; ++y) kq[i][4 * f + y] = z[y];
        }
      }
    }
    there = has_page(pg.p.page) && key0 + lane < k_hi && lane < KT;
    if constexpr (Q4) {
      const uint32_t* p = kpbase + (has_page(pg.p.page) ? pg.p.page : 0) * ca.k.psp + (pg.p.slot + (RUN ? n : 0)) * ca.k.pss;
      if constexpr (NG == 4) {
        const u32x4 z = *(const u32x4*)p;
#pragma unroll
        for (int g = 0; g < 4; ++g) kpq[g] = z[g];
      } else if constexpr (NG == 2) {
        const u32x2 z = *(const u32x2*)p;
        kpq[0] = z[0];
        kpq[1] = z[1];
      } else {
        kpq[0] = *p;
      }
    }
  };

  // Rows r0 .. of the run's head to the LDS.
  auto stage = [&](int r0) {
    const int32_t* pos_b = a.positions + b * a.pos_stride;
    const int rows = ka.held * ROWS, t_first = fast_quot(ka.group, r0);
    if (rope) {
      const int t_last = fast_quot(ka.group, min(r0 + rows, ka.rows) - 1);
      const int32_t* rpos_b = a.rope_positions + b * a.pos_stride;
      if (lane < a.rope.rot / 2) {
        for (int tk = t_first + wave; tk <= t_last; tk += kWaves) {
          float co, si;
          turn_cos_sin(rate, rpos_b[tk], co, si);
          scs[tk - t_first][lane] = make_float2(co * a.rope.scale, si * a.rope.scale);
        }
      }
      __syncthreads();
    }
    for (int e = tid; e < rows * (D / 8); e += kThreads) {
      const int rl = e / (D / 8), piece = e % (D / 8), d0 = 8 * piece;
      const int r = min(r0 + rl, ka.rows - 1), tk = fast_quot(ka.group, r), hq = h * group + (r - tk * group);
      const T* src = (const T*)a.q.ptr + b * a.q.sb + hq * a.q.sh + tk * a.q.ss;
      if (piece == 0) {
        const float lse = ka.a.lse[((int64_t)b * a.heads_q + hq) * a.tokens + tk];
        srow[rl].lse = lse;
        // (a row without keys, and one beyond the rows, sees none)
        srow[rl].last = r0 + rl < ka.rows && lse != -INFINITY ? min(pos_b[tk], ka.capacity - 1) : -1;
      }
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
        rotate8(a.rope, scs[tk - t_first], d0, y, z);
      }
      const int cb = rl / ROWS, at = rl % ROWS * PACK;
      if constexpr (F32) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
          sq[cb][0][d0 / 16][(d0 % 16 / 4 + f) * 16 + at] =
              u32x4{__float_as_uint(y[4 * f]), __float_as_uint(y[4 * f + 1]), __float_as_uint(y[4 * f + 2]),
                    __float_as_uint(y[4 * f + 3])};
      } else {
        if constexpr (Q4) {
          const float lo = (y[0] + y[1]) + (y[2] + y[3]), hi = (y[4] + y[5]) + (y[6] + y[7]);
          float sgn = lo - hi, all = lo + hi;
          sgn = dpp_add<0xb1>(sgn), all = dpp_add<0xb1>(all);
          sgn = dpp_add<0x4e>(sgn), all = dpp_add<0x4e>(all);
          if constexpr (D / NGX == 64) sgn = dpp_add<0x141>(sgn), all = dpp_add<0x141>(all);
          if (d0 % (D / NGX) == 0) srow[rl].sum[d0 / (D / NGX)] = make_float2(sgn, all * 0.0625f);
          const float s8[8] = {y[0], -y[4], y[1], -y[5], y[2], -y[6], y[3], -y[7]};
#pragma unroll
          for (int f = 0; f < 8; ++f) y[f] = s8[f];
        }
        bf16x8 parts[QP];
        split<QP>(y, parts);
        // keys' quarters as they are: lane 16 j + row holds elements D / 4 j ..; else, of step i, elements 32 i + 8 j ..
        constexpr bool QUARTERS = Q4 && !ALIGNED;
        const int step = QUARTERS ? piece % STEPS : piece / 4, lane_j = QUARTERS ? piece / STEPS : piece % 4;
#pragma unroll
        for (int part = 0; part < QP; ++part)
#pragma unroll
          for (int f = 0; f < PACK; ++f) {  // (0 but in the pairs of the piece's group, where the pairs hold all groups)
            const bool own = !Q4 || NPH > 1 || d0 / (D / NGX) == f;
            sq[cb][part][step][16 * lane_j + at + f] = own ? __builtin_bit_cast(u32x4, parts[part]) : u32x4{0, 0, 0, 0};
          }
      }
    }
  };

  while (x < x_end) {
    // ---- a run of one head's units [u0, u1)
    const int u1 = min(row_units, u0 + (x_end - x));
    const int k_lo = u0 << ka.unit_shift;
    k_hi = min(len, u1 << ka.unit_shift);
    last_page = fast_quot(ca.table.page, k_hi - 1);
    kbase = (const char*)ca.k.data + h * ka.ksh;
    kpbase = Q4 ? ca.k.params + h * ca.k.psh : nullptr;
    table = ca.table.ptr + b * ca.table.stride;
    int key0 = k_lo + wave * KT;
    {
      const Pages pg = pages(key0);
      load(pg, key0);
    }
    Pages pn = pages(key0 + kWaves * KT);
    // (all wavefronts take as many turns: the rows of one are staged by all)
    for (int base = k_lo; base < k_hi; base += kWaves * KT) {
      const uint64_t exist = __ballot(there);
      if constexpr (Q4) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          sks[wave][lane][g] = __uint_as_float(kpq[g] << 16);
          skm[wave][lane][g] = __uint_as_float(kpq[g] & 0xffff0000u);
        }
        __builtin_amdgcn_wave_barrier();
        if constexpr (ALIGNED)
#pragma unroll
          for (int i = 0; i < SUB; ++i) by_channels(kq[i]);
      }
      float sum[SUB];
#pragma unroll
      for (int i = 0; i < SUB; ++i) sum[i] = 0.f;
      for (int cb0 = 0; cb0 < ka.blocks; cb0 += ka.held) {
        if (ka.blocks > ka.held || base == k_lo) {
          __syncthreads();
          stage(cb0 * ROWS);
          __syncthreads();
        }
        for (int cb = cb0; cb < min(cb0 + ka.held, ka.blocks); ++cb) {
          const typename S::Row* rows = srow + (cb - cb0) * ROWS + RV * j;  // the lane's
          // S: s[i][v] is key key0 + 16 i + n of row RV j + v
          float s[SUB][RV];
          if constexpr (Q4) {
#pragma unroll
            for (int ph = 0; ph < NPH; ++ph) {
              f32x4 y[SUB], all;
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float2 q2 = rows[r / PACK].sum[ph * PACK + r % PACK];
                all[r] = q2.y;
#pragma unroll
                for (int i = 0; i < SUB; ++i) y[i][r] = BF ? -kMid * q2.x : 0.f;  // (fp32: the codes are centred)
              }
#pragma unroll
              for (int f = ph * (STEPS / NPH); f < (ph + 1) * (STEPS / NPH); ++f) {
                bf16x8 k8[SUB];
#pragma unroll
                for (int i = 0; i < SUB; ++i) k8[i] = open(kq[i][f]);
#pragma unroll
                for (int part = QP - 1; part >= 0; --part) {
                  const u32x4 q = sq[cb - cb0][part][f][lane];
#pragma unroll
                  for (int i = 0; i < SUB; ++i)
                    y[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q), k8[i], y[i], 0, 0, 0);
                }
              }
#pragma unroll
              for (int i = 0; i < SUB; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  const int g = ph * PACK + r % PACK;
                  float& to = s[i][r / PACK];
                  const float z = skm[wave][16 * i + n][g] * all[r];
                  to = fmaf(sks[wave][16 * i + n][g], y[i][r], ph == 0 && r % PACK == 0 ? z : to + z);
                }
            }
          } else {
            constexpr int SUMS = F32 ? 2 : 1;  // (partial sums of an fp32 score: one chain rounds off twice as far)
            f32x4 y[SUMS][SUB];
#pragma unroll
            for (int z = 0; z < SUMS; ++z)
#pragma unroll
              for (int i = 0; i < SUB; ++i) y[z][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int part = QP - 1; part >= 0; --part)
#pragma unroll
              for (int f = 0; f < STEPS; ++f) {
                const u32x4 q = sq[cb - cb0][part][f][lane];
#pragma unroll
                for (int i = 0; i < SUB; ++i) {
                  const u32x4 k4 = {kq[i][4 * f], kq[i][4 * f + 1], kq[i][4 * f + 2], kq[i][4 * f + 3]};
                  if constexpr (BF) {
                    y[0][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q),
                                                                      __builtin_bit_cast(bf16x8, k4), y[0][i], 0, 0, 0);
                  } else {
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                      y[z % SUMS][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[z]), __uint_as_float(k4[z]),
                                                                            y[z % SUMS][i], 0, 0, 0);
                  }
                }
              }
#pragma unroll
            for (int i = 0; i < SUB; ++i)
#pragma unroll
              for (int v = 0; v < RV; ++v) s[i][v] = F32 ? y[0][i][v] + y[SUMS - 1][i][v] : y[0][i][v];
          }
          if (cb == ka.blocks - 1) {  // the tile's keys are done with: the next one's, and the pages after that
            load(pn, key0 + kWaves * KT);
            pn = pages(key0 + 2 * kWaves * KT);
          }
          int least = 0x7fffffff, last[RV];
#pragma unroll
          for (int v = 0; v < RV; ++v) {
            last[v] = rows[v].last;
            least = min(least, last[v]);
          }
          const bool all_see = exist == (KT == 64 ? ~0ull : (1ull << KT % 64) - 1) && __ballot(least < key0 + KT - 1) == 0;
          if (all_see) {
#pragma unroll
            for (int v = 0; v < RV; ++v) {
              const float lse = rows[v].lse;
#pragma unroll
              for (int i = 0; i < SUB; ++i) sum[i] += power(s[i][v], lse);
            }
          } else {
#pragma unroll
            for (int v = 0; v < RV; ++v) {
              const float lse = rows[v].lse;
#pragma unroll
              for (int i = 0; i < SUB; ++i) {
                const bool sees = (exist >> (16 * i + n) & 1) && key0 + 16 * i + n <= last[v];
                const float p = power(s[i][v], lse);
                sum[i] += sees ? p : 0.f;
              }
            }
          }
        }
      }
      // the quads' rows together; quad i takes sub-tile i's keys
      float own = 0.f;
#pragma unroll
      for (int i = 0; i < SUB; ++i) {
        const float y = column_sum(sum[i]);
        own = j == i ? y : own;
      }
      const int key = key0 + lane;
      if (lane < KT && key < k_hi) {
        const float* in = ka.a.in + b * ka.a.isb + h * ka.a.ish + key;
        ka.a.out[b * ka.a.osb + h * ka.a.osh + key] = ka.a.decay != 0.f ? fmaf(ka.a.decay, *in, own) : own;
      }
      key0 += kWaves * KT;
    }
    // ---- the next run
    x += u1 - u0;
    u0 = u1;
    if (u0 == row_units) {
      u0 = 0;
      if (++h == items) {
        h = 0;
        while (x < x_end) {  // (sequences without keys have no units)
          len = __builtin_amdgcn_readfirstlane(length_of(ka, ++b));
          row_units = units_of(ka, len);
          if (row_units > 0) break;
        }
      }
    }
  }
}

template <typename T, int D, int NG, int PACK, int QP>
hipError_t launch(KernelArgs& k, hipStream_t s) {
  using S = Shape<T, D, NG, PACK, QP>;
  constexpr int kWaves = S::THREADS / kWave;
  k.unit_shift = S::UNIT_SHIFT;
  const int64_t heads = (int64_t)k.a.q.batch * k.a.q.cache.heads_kv;
  auto units = [&]() -> int64_t { return ((int64_t)k.capacity + ((int64_t)1 << k.unit_shift) - 1) >> k.unit_shift; };
  while ((units() + 1) * heads > (1 << 30)) ++k.unit_shift;
  k.blocks = (k.rows + S::ROWS - 1) / S::ROWS;
  k.held = std::min(k.blocks, S::MOST);
  // as many workgroups as the GPU holds at once: by registers, and by the LDS
  const int lds = k.held * S::BYTES + (S::Q4 ? kWaves * S::KT * NG * 8 : 0);
  const int per_cu = std::max(1, std::min(S::WAVES * 4 / kWaves, (160 << 10) / (lds + 1024)));
  const dim3 grid((unsigned)std::min((int64_t)256 * per_cu, units() * heads));
  const size_t room = (size_t)k.held * S::BYTES;
  // whole aligned runs of 16 keys, their rows within 2^30 bytes, are looked up once (a rotated token after 131072 tokens: pages of 64
  // and 16 27 us, pages of 24, key by key, 29)
  const int64_t far = (int64_t)1 << 26;
  auto kernel = k.a.q.cache.table.page.d % 16 == 0 && k.kss < far ? weights_kernel<T, D, NG, PACK, QP, true>
                                                                 : weights_kernel<T, D, NG, PACK, QP, false>;
  if (lds > 64 << 10) {
    // (the kernel's, not the call's: every call sets the same, as others may be between theirs and their launch)
    const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::MOST * S::BYTES);
    if (e != hipSuccess) return e;
  }
  kernel<<<grid, S::THREADS, room, s>>>(k);
  return hipGetLastError();
}
template <typename T, int D, int NG, int PACK>
hipError_t launch(KernelArgs& k, hipStream_t s) {
  if constexpr (sizeof(T) == 4) return launch<T, D, NG, PACK, NG == 0 ? 1 : 3>(k, s);
  else return k.a.q.rope.freq ? launch<T, D, NG, PACK, 3>(k, s) : launch<T, D, NG, PACK, 1>(k, s);
}
// (the groups share the operand's rows where these leave room for all of them: the keys are opened once then)
template <typename T, int D, int NG>
hipError_t launch(KernelArgs& k, hipStream_t s) {
  if constexpr (NG > 1)
    if (k.rows <= 16 / NG) return launch<T, D, NG, NG>(k, s);
  return launch<T, D, NG, 1>(k, s);
}
template <typename T, int D>
hipError_t launch(KernelArgs& k, hipStream_t s) {
  const int group = k.a.q.cache.group;
  return group == 0 ? launch<T, D, 0>(k, s) : group == 32 ? launch<T, D, D / 32>(k, s) : launch<T, D, D / 64>(k, s);
}

}  // namespace

hipError_t launch_weights(const WeightArgs& a, hipStream_t s) {
  const QueryArgs& q = a.q;
  const bool q4 = q.cache.group != 0;
  KernelArgs k;
  k.a = a;
  const int size = q4 ? 1 : q.bf16 ? 2 : 4;
  k.ksp = q.cache.k.sp * size;
  k.ksh = q.cache.k.sh * size;
  k.kss = q.cache.k.ss * size;
  const int group = q.heads_q / q.cache.heads_kv;
  k.group = fast_div(group);
  k.rows = group * q.tokens;
  k.capacity = std::min(q.cache.table.max_pages * q.cache.table.page.d, a.width);
  k.scale = q.scale * (q4 ? 16.f : 1.f);
  if (q.bf16) return q.cache.head_dim == 128 ? launch<uint16_t, 128>(k, s) : launch<uint16_t, 64>(k, s);
  return q.cache.head_dim == 128 ? launch<float, 128>(k, s) : launch<float, 64>(k, s);
}

}  // namespace seer
