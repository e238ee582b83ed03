// paged_join.h -- the second launch of attention over a paged cache, which joins the partial results of rows that
// several workgroups shared.
#pragma once

#include <algorithm>

#include "paged_common.h"

namespace seer {
namespace {

constexpr int kWorkers = 512;  // workgroups of the first launch at most: two for each CU

struct JoinArgs {
  const int2* record;    // [batch heads_kv row_blocks] first slot and last workgroup of a split row, or -1
  const float2* part_ml; // [2 kWorkers][rows_block] maximum and sum
  const float* part_o;   // [2 kWorkers][rows_block][D]
  void* o;
  int64_t osb, osh, oss;
  float* lse;
  FastDiv group, blocks; // by the query heads of a KV head and row_blocks
  int batch, heads_q, heads_kv, tokens;
  int rows, row_blocks, rows_block;  // query rows of a KV head, their blocks, rows of a block
  float scale_log2;
};

// Rows whose keys several workgroups shared: their partial results, in the order of the keys.  A workgroup joins JR
// rows of an item, a wavefront forming the weights of a row (or part of one: all four then form the same); a thread sums
// 4 features over the parts grp, grp + GRP, ..  Four rows a workgroup keep a large batch's launch short, one row leaves
// fewer parts to each thread where the call has few rows (a token after 131072 tokens, 32 rows of 64 parts: 6.9 -> 4.8 us).
constexpr int kJoinThreads = 256;
template <typename T, int D, int JR>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(JoinArgs a) {
  constexpr int V4 = D / 4, GRP = kJoinThreads / (V4 * JR), AHEAD = 8, OWN = kWorkers / kWave;
  __shared__ float sW[JR][kWorkers];
  __shared__ float2 sT[JR];
  __shared__ __attribute__((aligned(16))) float sO[GRP][JR][D];
  asm volatile("" ::"s"(a.osb), "s"(a.lse), "s"(a.heads_q), "s"(a.rows), "s"(a.part_o));  // (every line of the arguments, now)
  const int2 rec = a.record[blockIdx.x];
  if (rec.x < 0) return;
  const int items = a.heads_kv * a.row_blocks;
  const int b = blockIdx.x / (uint32_t)items, item = blockIdx.x - b * items;
  const int h = fast_quot(a.blocks, item), rb = item - h * a.row_blocks;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int nrows = min(a.rows_block, a.rows - rb * a.rows_block);
  const int w0 = rec.x / 2, parts = rec.y - w0 + 1;
  auto slot = [&](int p, int rl) { return (int64_t)(p == 0 ? rec.x : 2 * (w0 + p)) * a.rows_block + rl; };
  const float c = a.scale_log2;

  // the first parts are on their way while the weights are formed
  const int wrow = wave % JR;
  const int row = min((int)blockIdx.y * JR + wrow, nrows - 1);
  float2 ml[OWN];
#pragma unroll
  for (int i = 0; i < OWN; ++i)
    if (i * kWave < parts) ml[i] = a.part_ml[slot(min(lane + i * kWave, parts - 1), row)];
  const int d = tid % V4 * 4, jr = tid / V4 % JR, grp = tid / (V4 * JR);
  const int rl = min((int)blockIdx.y * JR + jr, nrows - 1);
  auto part = [&](int p) { return *(const f32x4*)(a.part_o + slot(p, rl) * D + d); };
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
  const int r = rb * a.rows_block + rl, t = fast_quot(a.group, r), hq = h * a.group.d + (r - t * a.group.d);
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

template <typename T, int D>
hipError_t launch_join(const JoinArgs& a, hipStream_t s) {
  const int64_t all = (int64_t)a.batch * a.heads_kv * a.row_blocks;
  const int rows = std::min(a.rows, a.rows_block);
  if (all * rows <= 2 * kWorkers)
    paged_join_kernel<T, D, 1><<<dim3((unsigned)all, (unsigned)rows), kJoinThreads, 0, s>>>(a);
  else
    paged_join_kernel<T, D, 4><<<dim3((unsigned)all, (unsigned)((rows + 3) / 4)), kJoinThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace
}  // namespace seer
