// weights_kernels.hip -- the attention weight that each cached key gets from some queries (seer_kv_weights).
//
//   out[t] = decay in[t] + sum over the rows r that see t of exp(scale q_r . k_t - lse_r)
//
// The half of attention that needs no running maximum: the rows' log-sum-exps are known, so that a key's sum is
// its own affair.  A wavefront holds 64 keys (32 of fp32) as the operand of S^T = K Q^T and goes through the
// rows, 16 columns at a time; a lane adds up the weights of its keys over its columns, and the 16 columns are joined at the
// end.  So the keys are read once however many rows there are, a key belongs to one wavefront, and there are no
// atomics.  Few rows (a step of generation) are bound by reading K, many (the last tokens of a prompt) by the
// exponentials.
//
// Units of keys are dealt out to the workgroups as in attention, and keys in 4 bits enter as there
// (q4_attn_kernels.hip).
#include <algorithm>

#include "cache.h"
#include "q4_open.h"

namespace seer {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kWorkers = 512;  // workgroups at most: two for each CU

struct KernelArgs {
  WeightArgs a;
  int64_t ksp, ksh, kss;  // K's strides in bytes
  int rows;               // G tokens
  FastDiv group;
  int capacity;           // keys that are counted at most
  int unit_shift;         // log2 of the keys per unit
  float scale_log2;       // of a score (4 bits: of a score / 16)
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

// T: type of q, and of the keys where NG is 0 (else: 4 bits, NG groups of a head, PACK of them sharing the columns).
// QP: bf16 parts of q.  RUN: pages hold whole aligned runs of the keys of a lane.
template <typename T, int D, int NG, int PACK, int QP, bool RUN>
__global__ __launch_bounds__(kThreads, 2) void weights_kernel(KernelArgs ka) {
  constexpr bool BF = sizeof(T) == 2, Q4 = NG != 0, F32 = !BF && !Q4;
  constexpr int SUB = F32 ? 2 : 4;              // sub-tiles of 16 keys
  constexpr int PK = 4 * SUB;                   // keys of a lane
  constexpr int KT = 16 * SUB;
  constexpr int ROWS = 16 / PACK;               // rows of a column block
  constexpr int CB = PACK > 1 ? 1 : QP == 3 ? 2 : 4;  // column blocks that are in the LDS together
  constexpr int NPH = Q4 ? NG / PACK : 1;
  constexpr int STEPS = F32 ? D / 16 : D / 32;  // 16-byte pieces of Q^T per lane
  constexpr int KW = Q4 ? D / 32 : 4 * STEPS;   // dwords of a key per lane
  constexpr int NGX = Q4 ? NG : 1;
  constexpr bool TURNS = QP == 3 || F32;        // q may be rotated here
  __shared__ u32x4 sq[QP][CB][STEPS][kWave];
  __shared__ float2 scs[TURNS ? CB * ROWS : 1][D / 2];
  __shared__ float2 ssum[CB * ROWS][NGX];       // as in q4_attn_kernel
  __shared__ float slse[CB * ROWS];
  __shared__ int slast[CB * ROWS];
  __shared__ __attribute__((aligned(16))) uint32_t skp[kWaves][4][NGX][16];

  const QueryArgs& a = ka.a.q;
  const CacheArgs& ca = a.cache;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane % 16, j = lane / 16;  // column, run of PK keys
  const int gp = n / ROWS, row = n % ROWS;
  const int items = ca.heads_kv;
  const int group = ka.group.d;
  const float c = ka.scale_log2;
  const bool rope = TURNS && a.rope.freq != nullptr;
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
  const int w = blockIdx.x;
  if ((uint32_t)w >= total) return;  // (a share each at least, or none)
  const Deal deal(total, gridDim.x);
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

  // Keys' operand: lane row n of sub-tile i is key PK (n / 4) + 4 i + n % 4 of a tile.
  const int kk = n / 4 * PK + n % 4;
  int k_hi;
  const char* kbase;
  const uint32_t* kpbase;
  const int32_t* table;
  uint32_t kq[SUB][KW];
  uint32_t kpq[NGX];
  bool there;  // key `lane` of the tile is counted and its page exists
  // Page of a key (-1: none) and slot, for places that are read: the pool's first slots where there is none.
  struct At {
    int page, slot;
    bool ok;
  };
  auto place = [&](int key) -> At {
    const int i = fast_quot(ca.table.page, max(min(key, k_hi - 1), 0));
    const int page = table[i];
    const bool ok = key < k_hi && (uint32_t)page < (uint32_t)ca.table.num_pages;
    return {ok ? page : 0, ok ? key - i * ca.table.page.d : 0, ok};
  };
  auto load = [&](int key0) {
    const char* run = nullptr;
    if constexpr (RUN) {  // (the run's first key: it exists where any of them does)
      const At s = place(key0 + n / 4 * PK);
      run = kbase + s.page * ka.ksp + (s.slot + n % 4) * ka.kss;
    }
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
      const char* p;
      if constexpr (RUN) {
        p = run + 4 * i * ka.kss;
      } else {
        const At s = place(key0 + kk + 4 * i);
        p = kbase + s.page * ka.ksp + s.slot * ka.kss;
      }
      if constexpr (KW == 2) {
        const u32x2 z = *(const u32x2*)p;
        kq[i][0] = z[0];
        kq[i][1] = z[1];
      } else {
#pragma unroll
        for (int f = 0; f < KW / 4; ++f) {
          const u32x4 z = *(const u32x4*)(p + 64 * f);
#pragma unroll
          for (int y = 0; y < 4; ++y) kq[i][4 * f + y] = z[y];
        }
      }
    }
    const int key = key0 + min(lane, KT - 1);
    const At s = place(key);
    there = s.ok && lane < KT;
    if constexpr (Q4) {
      const uint32_t* p = kpbase + s.page * ca.k.psp + s.slot * ca.k.pss;
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
  const int blocks = (ka.rows + ROWS - 1) / ROWS;  // of columns
  auto stage = [&](int r0) {
    const int32_t* pos_b = a.positions + b * a.pos_stride;
    const int t_first = fast_quot(ka.group, r0);
    if (rope) {
      const int t_last = fast_quot(ka.group, min(r0 + CB * ROWS, ka.rows) - 1);
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
    for (int e = tid; e < CB * ROWS * (D / 8); e += kThreads) {
      const int rl = e / (D / 8), piece = e % (D / 8), d0 = 8 * piece;
      const int r = min(r0 + rl, ka.rows - 1), tk = fast_quot(ka.group, r), hq = h * group + (r - tk * group);
      const T* src = (const T*)a.q.ptr + b * a.q.sb + hq * a.q.sh + tk * a.q.ss;
      if (piece == 0) {
        const float lse = ka.a.lse[((int64_t)b * a.heads_q + hq) * a.tokens + tk];
        slse[rl] = lse * kLog2e;
        // (a row without keys, and one beyond the rows, sees none)
        slast[rl] = r0 + rl < ka.rows && lse != -INFINITY ? min(pos_b[tk], ka.capacity - 1) : -1;
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
      const int cb = rl / ROWS, col = rl % ROWS;
      if constexpr (F32) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
          sq[0][cb][d0 / 16][(d0 % 16 / 4 + f) * 16 + col] =
              u32x4{__float_as_uint(y[4 * f]), __float_as_uint(y[4 * f + 1]), __float_as_uint(y[4 * f + 2]),
                    __float_as_uint(y[4 * f + 3])};
      } else {
        float s8[8];
        if constexpr (Q4) {
          const float lo = (y[0] + y[1]) + (y[2] + y[3]), hi = (y[4] + y[5]) + (y[6] + y[7]);
          float sgn = lo - hi, all = lo + hi;
          sgn = dpp_add<0xb1>(sgn), all = dpp_add<0xb1>(all);
          sgn = dpp_add<0x4e>(sgn), all = dpp_add<0x4e>(all);
          if constexpr (D / NGX == 64) sgn = dpp_add<0x141>(sgn), all = dpp_add<0x141>(all);
          if (d0 % (D / NGX) == 0) ssum[rl][d0 / (D / NGX)] = make_float2(sgn, all * 0.0625f);
#pragma unroll
          for (int f = 0; f < 4; ++f) {
            s8[2 * f] = y[f];
            s8[2 * f + 1] = -y[4 + f];
          }
        } else {
#pragma unroll
          for (int f = 0; f < 8; ++f) s8[f] = y[f];
        }
        // 4 bits: lane 16 j + col holds elements D / 4 j ..; else, of step i, elements 32 i + 8 j ..
        const int step = Q4 ? piece % STEPS : piece / 4, lane_j = Q4 ? piece / STEPS : piece % 4;
        if constexpr (QP == 3) {
          bf16x8 z3[3];
          split3(s8, z3);
#pragma unroll
          for (int part = 0; part < 3; ++part)
#pragma unroll
            for (int f = 0; f < PACK; ++f) {  // (0 but in the columns of the piece's group)
              const bool own = PACK == 1 || piece * 8 / (D / NGX) == f;
              u32x4 y4 = __builtin_bit_cast(u32x4, z3[part]);
              if (!own) y4 = u32x4{0, 0, 0, 0};
              sq[part][cb][step][16 * lane_j + f * ROWS + col] = y4;
            }
        } else {
          u32x4 z1;
#pragma unroll
          for (int f = 0; f < 4; ++f)
            z1[f] = __builtin_amdgcn_perm(__float_as_uint(s8[2 * f + 1]), __float_as_uint(s8[2 * f]), 0x07060302u);
#pragma unroll
          for (int f = 0; f < PACK; ++f) {
            const bool own = PACK == 1 || piece * 8 / (D / NGX) == f;
            sq[0][cb][step][16 * lane_j + f * ROWS + col] = own ? z1 : u32x4{0, 0, 0, 0};
          }
        }
      }
    }
  };

  while (x < x_end) {
    // ---- a run of one head's units [u0, u1)
    const int u1 = min(row_units, u0 + (x_end - x));
    k_hi = min(len, u1 << ka.unit_shift);
    kbase = (const char*)ca.k.data + h * ka.ksh + (Q4 ? 4 * KW : 16) * j;
    kpbase = Q4 ? ca.k.params + h * ca.k.psh : nullptr;
    table = ca.table.ptr + b * ca.table.stride;
    int key0 = (u0 << ka.unit_shift) + wave * KT;
    load(key0);
    // (all wavefronts take as many turns: the rows of one are staged by all)
    for (int base = u0 << ka.unit_shift; base < k_hi; base += kWaves * KT) {
      const bool has = key0 < k_hi;
      const uint32_t exist = (uint32_t)(__ballot(there) >> PK * j) & ((1u << PK) - 1u);
      if constexpr (Q4) {
#pragma unroll
        for (int g = 0; g < NG; ++g) skp[wave][j][g][n] = kpq[g];
        __builtin_amdgcn_wave_barrier();
      }
      float sum[PK];
#pragma unroll
      for (int e = 0; e < PK; ++e) sum[e] = 0.f;
      for (int cb0 = 0; cb0 < blocks; cb0 += CB) {
        if (blocks > CB || base == u0 << ka.unit_shift) {
          __syncthreads();
          stage(cb0 * ROWS);
          __syncthreads();
        }
        for (int cb = cb0; cb < min(cb0 + CB, blocks); ++cb) {
          const int col = (cb - cb0) * ROWS + row;
          // S^T: element e is key key0 + PK j + e of the lane's column
          float s[PK];
          if constexpr (Q4) {
#pragma unroll
            for (int e = 0; e < PK; ++e) s[e] = 0.f;
            const int quad_group = j * NG / 4;
#pragma unroll
            for (int ph = 0; ph < NPH; ++ph) {
              const uint32_t own = quad_group == ph ? ~0u : 0u;
              const float2 qsum = ssum[col][ph * PACK + gp];
              u32x4 kp[4];
#pragma unroll
              for (int f = 0; f < 4; ++f) kp[f] = *(const u32x4*)&skp[wave][j][ph * PACK + gp][4 * f];
              const float y0 = -kMid * qsum.x;
              f32x4 y[SUB];
#pragma unroll
              for (int i = 0; i < SUB; ++i) y[i] = f32x4{y0, y0, y0, y0};
#pragma unroll
              for (int part = QP - 1; part >= 0; --part)
#pragma unroll
                for (int f = 0; f < STEPS; ++f) {
                  u32x4 q = sq[part][cb - cb0][f][lane];
                  if constexpr (NPH > 1)
#pragma unroll
                    for (int z = 0; z < 4; ++z) q[z] &= own;
#pragma unroll
                  for (int i = 0; i < SUB; ++i)
                    y[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(open8(kq[i][f]), __builtin_bit_cast(bf16x8, q), y[i], 0, 0, 0);
                }
#pragma unroll
              for (int i = 0; i < SUB; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  const uint32_t p = kp[i][r];
                  s[4 * i + r] = fmaf(__uint_as_float(p << 16), y[i][r],
                                      fmaf(__uint_as_float(p & 0xffff0000u), qsum.y, s[4 * i + r]));
                }
            }
            if constexpr (PACK >= 2)
#pragma unroll
              for (int e = 0; e < PK; ++e) s[e] = dpp_add<0x128>(s[e]);  // row_ror 8
            if constexpr (PACK == 4)
#pragma unroll
              for (int e = 0; e < PK; ++e) s[e] = dpp_add<0x124>(s[e]);  // row_ror 4
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
                const u32x4 q = sq[part][cb - cb0][f][lane];
#pragma unroll
                for (int i = 0; i < SUB; ++i) {
                  const u32x4 k4 = {kq[i][4 * f], kq[i][4 * f + 1], kq[i][4 * f + 2], kq[i][4 * f + 3]};
                  if constexpr (BF) {
                    y[0][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k4),
                                                                      __builtin_bit_cast(bf16x8, q), y[0][i], 0, 0, 0);
                  } else {
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                      y[z % SUMS][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k4[z]), __uint_as_float(q[z]),
                                                                            y[z % SUMS][i], 0, 0, 0);
                  }
                }
              }
            if constexpr (F32)
#pragma unroll
              for (int i = 0; i < SUB; ++i) y[0][i] += y[1][i];
#pragma unroll
            for (int e = 0; e < PK; ++e) s[e] = y[0][e / 4][e % 4];
          }
          if (cb == blocks - 1) load(key0 + kWaves * KT);  // the tile's keys are done with
          const float lse = slse[col];
          const int last = slast[col] + 1 - (key0 + PK * j);
          const uint32_t seen = exist & ((1u << min(max(last, 0), PK)) - 1u);
#pragma unroll
          for (int e = 0; e < PK; ++e) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[e], c, -lse));
            sum[e] += seen >> e & 1 ? p : 0.f;
          }
        }
      }
      // the columns together; lane n of a run takes its key n
      float mine_e = 0.f;
#pragma unroll
      for (int e = 0; e < PK; ++e) {
        float y = sum[e];
        y = dpp_add<0x128>(y);
        y = dpp_add<0x124>(y);
        y = dpp_add<0x122>(y);
        y = dpp_add<0x121>(y);
        mine_e = n == e ? y : mine_e;
      }
      const int key = key0 + PK * j + n;
      if (has && n < PK && key < k_hi) {
        const float y = mine_e * (1.f / PACK);  // (the groups' columns hold the same weights)
        const float* in = ka.a.in + b * ka.a.isb + h * ka.a.ish + key;
        ka.a.out[b * ka.a.osb + h * ka.a.osh + key] = ka.a.decay != 0.f ? fmaf(ka.a.decay, *in, y) : y;
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
    __syncthreads();
  }
}

template <typename T, int D, int NG, int PACK, int QP>
hipError_t launch(const KernelArgs& k, dim3 grid, hipStream_t s) {
  constexpr int PK = sizeof(T) == 4 && NG == 0 ? 8 : 16;
  if (k.a.q.cache.table.page.d % PK == 0) weights_kernel<T, D, NG, PACK, QP, true><<<grid, kThreads, 0, s>>>(k);
  else weights_kernel<T, D, NG, PACK, QP, false><<<grid, kThreads, 0, s>>>(k);
  return hipGetLastError();
}
template <typename T, int D, int NG, int PACK>
hipError_t launch(const KernelArgs& k, dim3 grid, hipStream_t s) {
  if constexpr (sizeof(T) == 4 && NG == 0) {
    return launch<T, D, 0, 1, 1>(k, grid, s);
  } else {
    if constexpr (sizeof(T) == 2)
      if (!k.a.q.rope.freq) return launch<T, D, NG, PACK, 1>(k, grid, s);
    return launch<T, D, NG, PACK, 3>(k, grid, s);
  }
}
// (the groups share the columns where the rows leave room for all of them)
template <typename T, int D, int NG>
hipError_t launch(const KernelArgs& k, dim3 grid, hipStream_t s) {
  if constexpr (NG > 1)
    if (k.rows <= 16 / NG) return launch<T, D, NG, NG>(k, grid, s);
  return launch<T, D, NG, 1>(k, grid, s);
}
template <typename T, int D>
hipError_t launch(const KernelArgs& k, dim3 grid, hipStream_t s) {
  const int group = k.a.q.cache.group;
  return group == 0 ? launch<T, D, 0>(k, grid, s) : group == 32 ? launch<T, D, D / 32>(k, grid, s) : launch<T, D, D / 64>(k, grid, s);
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
  k.unit_shift = q4 || q.bf16 ? 8 : 7;
  const int64_t rows = (int64_t)q.batch * q.cache.heads_kv;
  auto units = [&]() -> int64_t { return ((int64_t)k.capacity + ((int64_t)1 << k.unit_shift) - 1) >> k.unit_shift; };
  while ((units() + 1) * rows > (1 << 30)) ++k.unit_shift;
  k.scale_log2 = q.scale * kLog2e * (q4 ? 16.f : 1.f);
  const dim3 grid((unsigned)std::min((int64_t)kWorkers, units() * rows));
  if (q.bf16) return q.cache.head_dim == 128 ? launch<uint16_t, 128>(k, grid, s) : launch<uint16_t, 64>(k, grid, s);
  return q.cache.head_dim == 128 ? launch<float, 128>(k, grid, s) : launch<float, 64>(k, grid, s);
}

}  // namespace seer
