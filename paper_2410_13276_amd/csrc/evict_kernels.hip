// evict_kernels.hip -- cutting a paged cache to the keys of the largest weight (seer_kv_evict).
//
// One workgroup for each sequence and KV head finds the slots that stay: a radix selection of the least weight
// that does (three passes over histograms of 11, 11 and 10 bits in the LDS), then one over the slots in
// their order, which counts, and one which writes.  A second launch moves the keys and values, 16 bytes a thread,
// whatever they are held as: the places it writes are no places that it reads, so that it needs no order.
#include <algorithm>

#include "cache.h"
#include "device_common.h"

namespace seer {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;

// Order of weights as that of integers: NaN above all.
__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? 0xffffffffu : ordered_key(w); }

struct SelectArgs2 {
  EvictArgs a;
  int capacity;  // slots that a table row has room for
};

// Sum over the workgroup of the waves' values before this wave's, and of all.
__device__ __forceinline__ int2 before(int mine, int* sh, int wave, int lane) {
  if (lane == 0) sh[wave] = mine;
  __syncthreads();
  int2 r = {0, 0};
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    r.x += i < wave ? sh[i] : 0;
    r.y += sh[i];
  }
  __syncthreads();
  return r;
}

__global__ __launch_bounds__(kThreads) void evict_select_kernel(SelectArgs2 ka) {
  const EvictArgs& a = ka.a;
  __shared__ int hist[kBins];
  __shared__ int shw[kWaves];
  __shared__ int found[2];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int b = blockIdx.x / (uint32_t)a.cache.heads_kv, h = blockIdx.x - b * a.cache.heads_kv;
  const float* weights = a.weights + b * a.sb + h * a.sh;
  float* new_weights = a.new_weights + b * a.nsb + h * a.nsh;
  int32_t* kept = a.kept + (int64_t)blockIdx.x * a.keep;
  const int n = min(max(a.lengths[b], 0), ka.capacity);
  const int taken = min(n, a.keep);
  auto weight = [&](int i) { return i < a.width ? weights[i] : 0.f; };

  if (h == 0 && tid == 0) a.new_lengths[b] = taken;
  for (int64_t i = taken + tid; i < a.new_width; i += kThreads) new_weights[i] = 0.f;
  for (int64_t i = taken + tid; i < a.keep; i += kThreads) kept[i] = -1;
  auto keep_slot = [&](int to, int slot) {
    kept[to] = slot;
    new_weights[to] = weight(slot);
  };
  if (n <= a.keep) {
    for (int i = tid; i < n; i += kThreads) keep_slot(i, i);
    return;
  }
  for (int i = tid; i < a.first; i += kThreads) keep_slot(i, i);
  for (int i = tid; i < a.last; i += kThreads) keep_slot(a.keep - a.last + i, n - a.last + i);
  const int lo = a.first, hi = n - a.last, want = a.keep - a.first - a.last;
  if (want == 0) return;

  // ---- the want-th largest key of [lo, hi): digit by digit from the top
  uint32_t prefix = 0;
  int left = want;  // of the keys that begin with `prefix`
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
    __syncthreads();
#pragma unroll 4
    for (int i = lo + tid; i < hi; i += kThreads) {
      const uint32_t key = weight_key(weight(i));
      if (pass == 0 || key >> (shift + bits) == prefix) atomicAdd(&hist[key >> shift & ((1u << bits) - 1)], 1);
    }
    __syncthreads();
    // thread t: bins 2 t and 2 t + 1 counted from the top
    const int c0 = hist[kBins - 1 - 2 * tid], c1 = hist[kBins - 2 - 2 * tid];
    int up = c0 + c1;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const int y = __shfl_up(up, d);
      if (lane >= d) up += y;
    }
    const int2 s = before(__shfl(up, kWave - 1), shw, wave, lane);
    const int above = s.x + up - c0 - c1;  // keys in higher bins than this thread's
    if (above < left && above + c0 + c1 >= left) {
      const bool first = above + c0 >= left;
      found[0] = kBins - (first ? 1 : 2) - 2 * tid;
      found[1] = left - above - (first ? 0 : c0);
    }
    __syncthreads();
    prefix = prefix << bits | (uint32_t)found[0];
    left = found[1];
    __syncthreads();
  }

  // ---- in order: a wavefront takes a run of slots, counts those above the key and those equal to it, and then
  // writes; of the equal ones the first `left` stay
  const int seg = ((hi - lo + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
  const int s0 = min(lo + wave * seg, hi), s1 = min(s0 + seg, hi);
  int above = 0, equal = 0;
#pragma unroll 4
  for (int i = s0; i < s1; i += kWave) {
    const int at = i + lane;
    const uint32_t key = at < s1 ? weight_key(weight(at)) : 0u;
    above += (int)__popcll(__ballot(at < s1 && key > prefix));
    equal += (int)__popcll(__ballot(at < s1 && key == prefix));
  }
  int above_at = before(above, shw, wave, lane).x, equal_at = before(equal, shw, wave, lane).x;
#pragma unroll 4
  for (int i = s0; i < s1; i += kWave) {
    const int at = i + lane;
    const float w = at < s1 ? weight(at) : 0.f;
    const uint32_t key = weight_key(w);
    const uint64_t gt = __ballot(at < s1 && key > prefix), eq = __ballot(at < s1 && key == prefix);
    const int eq_before = equal_at + (int)__popcll(eq & lanemask_lt());
    const bool stays = (gt >> lane & 1) || ((eq >> lane & 1) && eq_before < left);
    if (stays) {
      const int to = a.first + above_at + (int)__popcll(gt & lanemask_lt()) + min(eq_before, left);
      kept[to] = at;
      new_weights[to] = w;
    }
    above_at += (int)__popcll(gt);
    equal_at += (int)__popcll(eq);
  }
}

struct MoveArgs {
  EvictArgs a;
  int64_t entries;  // batch heads_kv keep
  int64_t ksp, ksh, kss, vsp, vsh, vss;  // strides in bytes
};

// LANES threads move an entry, each 16 bytes of its key and of its value; PARAMS: and a dword of their params.
template <int LANES, int PARAMS>
__global__ __launch_bounds__(256) void evict_move_kernel(MoveArgs ka) {
  const EvictArgs& a = ka.a;
  const int piece = threadIdx.x % LANES;
  const uint32_t keep = a.keep, heads = a.cache.heads_kv;
  for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES; e < ka.entries; e += (int64_t)gridDim.x * (256 / LANES)) {
    const int64_t pair = e / keep;
    const int to = (int)(e - pair * keep), b = (int)(pair / heads), h = (int)(pair - (int64_t)b * heads);
    const int from = a.kept[e];
    const int tp = fast_quot(a.to.page, to);
    const int to_page = a.to.ptr[b * a.to.stride + tp];
    if (from < 0) continue;
    const int fp = fast_quot(a.cache.table.page, from);
    const int from_page = a.cache.table.ptr[b * a.cache.table.stride + fp];
    if ((uint32_t)from_page >= (uint32_t)a.cache.table.num_pages || (uint32_t)to_page >= (uint32_t)a.cache.table.num_pages) continue;
    const int64_t fs = from - fp * a.cache.table.page.d, ts = to - tp * a.to.page.d;
    const u32x4 k = *(const u32x4*)((const char*)a.cache.k.data + from_page * ka.ksp + h * ka.ksh + fs * ka.kss + 16 * piece);
    const u32x4 v = *(const u32x4*)((const char*)a.cache.v.data + from_page * ka.vsp + h * ka.vsh + fs * ka.vss + 16 * piece);
    uint32_t kp = 0, vp = 0;
    if (piece < PARAMS) {
      kp = a.cache.k.params[from_page * a.cache.k.psp + h * a.cache.k.psh + fs * a.cache.k.pss + piece];
      vp = a.cache.v.params[from_page * a.cache.v.psp + h * a.cache.v.psh + fs * a.cache.v.pss + piece];
    }
    *(u32x4*)((char*)a.cache.k.data + to_page * ka.ksp + h * ka.ksh + ts * ka.kss + 16 * piece) = k;
    *(u32x4*)((char*)a.cache.v.data + to_page * ka.vsp + h * ka.vsh + ts * ka.vss + 16 * piece) = v;
    if (piece < PARAMS) {
      ((uint32_t*)a.cache.k.params)[to_page * a.cache.k.psp + h * a.cache.k.psh + ts * a.cache.k.pss + piece] = kp;
      ((uint32_t*)a.cache.v.params)[to_page * a.cache.v.psp + h * a.cache.v.psh + ts * a.cache.v.pss + piece] = vp;
    }
  }
}

template <int LANES, int PARAMS>
hipError_t move(const MoveArgs& m, hipStream_t s) {
  const int64_t blocks = (m.entries * LANES + 255) / 256;
  evict_move_kernel<LANES, PARAMS><<<(unsigned)std::min(blocks, (int64_t)1 << 22), 256, 0, s>>>(m);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
  SelectArgs2 k = {a, a.cache.table.max_pages * a.cache.table.page.d};
  const int64_t pairs = (int64_t)a.batch * a.cache.heads_kv;
  evict_select_kernel<<<(unsigned)pairs, kThreads, 0, s>>>(k);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int size = a.cache.group ? 1 : a.bf16 ? 2 : 4;
  const PoolView &kc = a.cache.k, &vc = a.cache.v;
  const MoveArgs m = {a, pairs * a.keep, kc.sp * size, kc.sh * size, kc.ss * size, vc.sp * size, vc.sh * size, vc.ss * size};
  if (!a.cache.group) {
    const int bytes = a.cache.head_dim * size;
    return bytes == 512 ? move<32, 0>(m, s) : bytes == 256 ? move<16, 0>(m, s) : move<8, 0>(m, s);
  }
  if (a.cache.head_dim == 128) return a.cache.group == 32 ? move<4, 4>(m, s) : move<4, 2>(m, s);
  return a.cache.group == 32 ? move<2, 2>(m, s) : move<2, 1>(m, s);
}

}  // namespace seer
