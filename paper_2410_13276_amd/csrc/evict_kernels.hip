// evict_kernels.hip -- cutting a paged cache to the keys of the largest weight (seer_kv_evict).
//
// Which slots stay is found by a radix selection of the least weight that does, as an integer of its order: three
// histograms of 11, 11 and 10 bits in the LDS, then one pass over the slots in their order, which writes those above the
// weight and the first ones equal to it.  A workgroup does that for a sequence and KV head, its slots in registers where they
// fit.  Long rows of few heads are cut into parts, a workgroup each: their histograms go to the workspace and a launch
// a digit adds them up (no atomics between workgroups); what the parts before a part write follows from
// the histograms too.  A last launch moves the keys and values, 16 bytes a thread, whatever they are held as: the places it
// writes are no places that it reads, so that it needs no order.
//
// Measured, one MI355X: 64 sequences of 1700 to 2400 slots cut to 2048 (8 heads of 128 in 4 bits) 15 us to choose, 57 to move 336
// MB at 5.9e12 bytes a second, the memory's rate; 131072 slots cut to 4096 (bf16) 41 us to choose, by launches and barriers (the
// weights are 4 MB; the digits' launches take 5.9, 9.8 and 9.8 us, the one that writes 15.6; equal addresses of the LDS, nearly all
// in the first, cost it 1.0e5 cycles over 64 workgroups, 0.7 us), 7.7 to move 34 MB. A row of 131072 slots by one workgroup a head
// takes 185 us to choose; what has more than 128 pairs is done so (64 sequences of 8 heads of 131072 slots cut to 1024: 389 us
// together, whose bytes take 164).
#include <algorithm>

#include "cache.h"
#include "device_common.h"

namespace seer {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;
// slots of a part of a long row at least (131072 slots of 8 heads, the four launches together: 42 us; 8192 40 to 41, 4096 48, as each adds
// up all parts' histograms)
constexpr int kPart = 16384;
// of a part in the workspace: three histograms; its slots above the weight by the first and second digit; (the first part's:)
// the weight's upper bits and how many stay of those that have them, after the first and the second digit
constexpr int kPartInts = 3 * kBins + 64;

// Order of weights as that of integers: NaN above all.
__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? 0xffffffffu : ordered_key(w); }

struct PickArgs {
  EvictArgs a;
  int capacity;  // slots that a table row has room for
  int parts;     // of a row
  int* hist;     // [pair][part][kPartInts]
};

constexpr int shift_of(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }
constexpr int bits_of(int digit) { return digit == 2 ? 10 : 11; }

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
__device__ __forceinline__ int wave_total(int x) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
  return x;
}

// The weight that is looked for, as far as it is known: its upper bits, and how many of those that have them stay.
struct Known {
  uint32_t prefix;
  int left;
};
// One digit more, from the counts c0 and c1 of bins 2 t and 2 t + 1 from the top of thread t.
__device__ __forceinline__ Known narrow(const Known& k, int c0, int c1, int bits, int* shw, int* found, int tid, int wave, int lane) {
  int up = c0 + c1;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int y = __shfl_up(up, d);
    if (lane >= d) up += y;
  }
  const int2 s = before(__shfl(up, kWave - 1), shw, wave, lane);
  const int above = s.x + up - c0 - c1;  // keys in higher bins than this thread's
  if (above < k.left && above + c0 + c1 >= k.left) {
    const bool first = above + c0 >= k.left;
    found[0] = kBins - (first ? 1 : 2) - 2 * tid;
    found[1] = k.left - above - (first ? 0 : c0);
  }
  __syncthreads();
  const Known r = {k.prefix << bits | (uint32_t)found[0], found[1]};
  __syncthreads();
  return r;
}

// A row of weights and what of it is chosen from: slots [lo, hi), of which `want` stay.
struct Row {
  const float* weights;
  float* new_weights;
  int32_t* kept;
  int n, taken, lo, hi, want;
};
__device__ __forceinline__ Row row_of(const PickArgs& ka, int pair) {
  const EvictArgs& a = ka.a;
  const int b = pair / (uint32_t)a.cache.heads_kv, h = pair - b * a.cache.heads_kv;
  Row r;
  r.weights = a.weights + b * a.sb + h * a.sh;
  r.new_weights = a.new_weights + b * a.nsb + h * a.nsh;
  r.kept = a.kept + (int64_t)pair * a.keep;
  r.n = min(max(a.lengths[b], 0), ka.capacity);
  r.taken = min(r.n, a.keep);
  r.lo = a.first;
  r.hi = r.n - a.last;
  r.want = r.n > a.keep ? a.keep - a.first - a.last : 0;
  return r;
}
// What needs no choice: the slots that always stay, and what is behind them.
__device__ __forceinline__ void write_rest(const PickArgs& ka, const Row& r, int tid) {
  const EvictArgs& a = ka.a;
  for (int64_t i = r.taken + tid; i < a.new_width; i += kThreads) r.new_weights[i] = 0.f;
  for (int64_t i = r.taken + tid; i < a.keep; i += kThreads) r.kept[i] = -1;
  auto keep_slot = [&](int to, int slot) {
    r.kept[to] = slot;
    r.new_weights[to] = slot < a.width ? r.weights[slot] : 0.f;
  };
  if (r.n <= a.keep) {
    for (int i = tid; i < r.n; i += kThreads) keep_slot(i, i);
    return;
  }
  for (int i = tid; i < a.first; i += kThreads) keep_slot(i, i);
  for (int i = tid; i < a.last; i += kThreads) keep_slot(a.keep - a.last + i, r.n - a.last + i);
}

// A workgroup's slots [lo, hi): a run for each wavefront, which takes EL at a time for each lane.
template <int EL>
struct Slots {
  const Row& r;
  int width, s0, s1, lane;
  bool held;  // they are in w
  float w[EL];
  __device__ __forceinline__ Slots(const Row& row, int width, int lo, int hi, int wave, int lane)
      : r(row), width(width), lane(lane) {
    const int seg = ((hi - lo + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
    s0 = min(lo + wave * seg, hi);
    s1 = min(s0 + seg, hi);
    held = s1 - s0 <= EL * kWave;
    if (held) fetch(s0);
  }
  __device__ __forceinline__ void fetch(int i0) {
#pragma unroll
    for (int f = 0; f < EL; ++f) {
      const int at = i0 + f * kWave + lane;
      w[f] = at < s1 && at < width ? r.weights[at] : 0.f;
    }
  }
  // use(slot, weight, whether there is one), in the slots' order by wavefronts; the lanes of a wavefront together
  template <typename Use>
  __device__ __forceinline__ void each(Use use) {
    for (int i0 = s0; i0 < s1; i0 += EL * kWave) {
      if (!held) fetch(i0);
#pragma unroll
      for (int f = 0; f < EL; ++f) {
        if (i0 + f * kWave >= s1) break;
        const int at = i0 + f * kWave + lane;
        use(at, w[f], at < s1);
      }
    }
  }
};

template <int EL>
__device__ __forceinline__ void count_digit(Slots<EL>& slots, const Known& k, int digit, int* hist, int tid) {
  const int shift = shift_of(digit), bits = bits_of(digit);
  for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
  __syncthreads();
  slots.each([&](int, float w, bool in) {
    const uint32_t key = weight_key(w);
    if (in && (digit == 0 || key >> (shift + bits) == k.prefix)) atomicAdd(&hist[key >> shift & ((1u << bits) - 1)], 1);
  });
  __syncthreads();
}

// The slots that stay to kept and new_weights, from place `above` + the equal ones taken before (`equal` are before).
template <int EL>
__device__ __forceinline__ void write_kept(Slots<EL>& slots, const Row& r, const Known& k, int above, int equal, int* shw, int wave,
                                           int lane) {
  int gts = 0, eqs = 0;
  slots.each([&](int, float w, bool in) {
    const uint32_t key = weight_key(w);
    gts += (int)__popcll(__ballot(in && key > k.prefix));
    eqs += (int)__popcll(__ballot(in && key == k.prefix));
  });
  above += before(gts, shw, wave, lane).x;
  equal += before(eqs, shw, wave, lane).x;
  slots.each([&](int at, float w, bool in) {
    const uint32_t key = weight_key(w);
    const uint64_t gt = __ballot(in && key > k.prefix), eq = __ballot(in && key == k.prefix);
    const int eq_before = equal + (int)__popcll(eq & lanemask_lt());
    if ((gt >> lane & 1) || ((eq >> lane & 1) && eq_before < k.left)) {
      const int to = r.lo + above + (int)__popcll(gt & lanemask_lt()) + min(eq_before, k.left);
      r.kept[to] = at;
      r.new_weights[to] = w;
    }
    above += (int)__popcll(gt);
    equal += (int)__popcll(eq);
  });
}

// A row whole.
template <int EL>
__global__ __launch_bounds__(kThreads) void evict_pick_kernel(PickArgs ka) {
  __shared__ int hist[kBins];
  __shared__ int shw[kWaves], found[2];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const Row r = row_of(ka, blockIdx.x);
  Slots<EL> slots(r, ka.a.width, r.lo, r.want ? r.hi : r.lo, wave, lane);
  write_rest(ka, r, tid);
  if (r.want == 0) return;
  Known k = {0, r.want};
#pragma unroll 1
  for (int digit = 0; digit < 3; ++digit) {
    count_digit(slots, k, digit, hist, tid);
    k = narrow(k, hist[kBins - 1 - 2 * tid], hist[kBins - 2 - 2 * tid], bits_of(digit), shw, found, tid, wave, lane);
  }
  write_kept(slots, r, k, 0, 0, shw, wave, lane);
}

// A part of a row: DIGIT's histogram of it, or (3) what of it stays.
template <int EL, int DIGIT>
__global__ __launch_bounds__(kThreads) void evict_part_kernel(PickArgs ka) {
  __shared__ int hist[kBins];
  __shared__ int shw[kWaves], found[2];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int part = blockIdx.x, pair = blockIdx.y;
  const Row r = row_of(ka, pair);
  if (DIGIT == 3 && part == 0) write_rest(ka, r, tid);
  if (r.want == 0) return;
  // (parts as long as this row asks for)
  const int each = max(kPart, (r.hi - r.lo + ka.parts - 1) / ka.parts);
  const int p0 = r.lo + part * each, p1 = min(p0 + each, r.hi), parts = (r.hi - r.lo + each - 1) / each;
  if (p0 >= r.hi) return;
  Slots<EL> slots(r, ka.a.width, p0, p1, wave, lane);
  int* all = ka.hist + (int64_t)pair * ka.parts * kPartInts;
  int* mine = all + part * kPartInts;
  Known k = {0, r.want};
  if constexpr (DIGIT > 0) {
    // the digit before, from all parts' histograms of it; what went before that stands behind the first part's
    constexpr int D0 = DIGIT - 1;
    const int b0 = kBins - 1 - 2 * tid, b1 = b0 - 1;
    int c0 = 0, c1 = 0, m0 = 0, m1 = 0;
    if (D0 > 0) k = {(uint32_t)all[3 * kBins + (D0 == 1 ? 3 : 5)], all[3 * kBins + (D0 == 1 ? 4 : 6)]};
#pragma unroll 8
    for (int i = 0; i < parts; ++i) {
      const int* h = all + i * kPartInts + D0 * kBins;
      const int x0 = h[b0], x1 = h[b1];
      if (i < part) m0 += x0, m1 += x1;
      c0 += x0;
      c1 += x1;
    }
    const int own0 = mine[D0 * kBins + b0], own1 = mine[D0 * kBins + b1];
    k = narrow(k, c0, c1, bits_of(D0), shw, found, tid, wave, lane);
    const int bin = (int)(k.prefix & ((1u << bits_of(D0)) - 1));
    if constexpr (DIGIT < 3) {
      // for the launches behind: the weight so far, and how many of the part's slots are above it by this digit
      const int above = before(wave_total((b0 > bin ? own0 : 0) + (b1 > bin ? own1 : 0)), shw, wave, lane).y;
      if (tid == 0) {
        mine[3 * kBins + D0] = above;
        if (part == 0) {
          // (a place for each digit's: a part of this launch may still read the one before)
          int* to = all + 3 * kBins + (D0 == 0 ? 3 : 5);
          to[0] = (int)k.prefix;
          to[1] = k.left;
        }
      }
    } else {
      // slots before this part's that are above the weight, and those equal to it
      int above = (b0 > bin ? m0 : 0) + (b1 > bin ? m1 : 0);
      if (tid < part) above += all[tid * kPartInts + 3 * kBins] + all[tid * kPartInts + 3 * kBins + 1];
      if (b0 == bin || b1 == bin) found[0] = b0 == bin ? m0 : m1;
      above = before(wave_total(above), shw, wave, lane).y;  // (its barriers also publish found)
      write_kept(slots, r, k, above, found[0], shw, wave, lane);
      return;
    }
  }
  if constexpr (DIGIT < 3) {
    count_digit(slots, k, DIGIT, hist, tid);
    for (int i = tid; i < kBins; i += kThreads) mine[DIGIT * kBins + i] = hist[i];
  }
}

struct MoveArgs {
  EvictArgs a;
  int64_t entries;  // batch heads_kv keep
  int capacity;
  int64_t ksp, ksh, kss, vsp, vsh, vss;  // strides in bytes
};

// LANES threads move an entry, each 16 bytes of its key and of its value; PARAMS: and a dword of their params.  (There are more
// threads than sequences.)
// PAST: past the caches, from 64 MiB on (8 heads of 128 in 4 bits, pages that no cache holds, selection included: 134 MB 87 -> 78
// us, 268 MB 168 -> 152; bf16 134 MB 62 -> 57, 268 MB 112 -> 101; 34 MB 23.8 -> 23.3, of 4 bits 30.5 -> 28.4).  What the caches may
// hold yet takes longer past them (17 MB of bf16 7.7 -> 9.1, a whole call of 67 MB 26 -> 31).
template <int LANES, int PARAMS, bool PAST>
__global__ __launch_bounds__(256) void evict_move_kernel(MoveArgs ka) {
  const EvictArgs& a = ka.a;
  const int piece = threadIdx.x % LANES;
  const uint32_t keep = a.keep, heads = a.cache.heads_kv;
  // the lengths, which may be written in place: the launches that read the old ones have ended
  if (const int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x; b < a.batch)
    a.new_lengths[b] = min(min(max(a.lengths[b], 0), ka.capacity), a.keep);
  auto fetch = [](const char* p) -> u32x4 {
    if constexpr (PAST) return __builtin_nontemporal_load((const u32x4*)p);
    else return *(const u32x4*)p;
  };
  auto put = [](char* p, const u32x4& x) {
    if constexpr (PAST) __builtin_nontemporal_store(x, (u32x4*)p);
    else *(u32x4*)p = x;
  };
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
    const u32x4 k = fetch((const char*)a.cache.k.data + from_page * ka.ksp + h * ka.ksh + fs * ka.kss + 16 * piece);
    const u32x4 v = fetch((const char*)a.cache.v.data + from_page * ka.vsp + h * ka.vsh + fs * ka.vss + 16 * piece);
    uint32_t kp = 0, vp = 0;
    if (piece < PARAMS) {
      kp = a.cache.k.params[from_page * a.cache.k.psp + h * a.cache.k.psh + fs * a.cache.k.pss + piece];
      vp = a.cache.v.params[from_page * a.cache.v.psp + h * a.cache.v.psh + fs * a.cache.v.pss + piece];
    }
    put((char*)a.cache.k.data + to_page * ka.ksp + h * ka.ksh + ts * ka.kss + 16 * piece, k);
    put((char*)a.cache.v.data + to_page * ka.vsp + h * ka.vsh + ts * ka.vss + 16 * piece, v);
    if (piece < PARAMS) {
      ((uint32_t*)a.cache.k.params)[to_page * a.cache.k.psp + h * a.cache.k.psh + ts * a.cache.k.pss + piece] = kp;
      ((uint32_t*)a.cache.v.params)[to_page * a.cache.v.psp + h * a.cache.v.psh + ts * a.cache.v.pss + piece] = vp;
    }
  }
}

// Parts of a row: as many as give the GPU work, of kPart slots or more.  256 workgroups: 128 rows of 131072 slots cut to 1024 take
// 165 us whole, 126 in 2 parts, 123 in 4; 256 rows 207 whole, 220 in 2 parts.  At most 32 parts: two rows of 1048576 slots 92 us in
// 16, 75 in 32, 81 in 64.  (The table's room counts, as the lengths are on the device: 3000 slots in a table of 131072 take 26 us,
// of 4096 14.)
int parts_of(int64_t pairs, int capacity) {
  return (int)std::max((int64_t)1, std::min({((int64_t)capacity + kPart - 1) / kPart, 256 / pairs, (int64_t)32}));
}

template <int LANES, int PARAMS>
hipError_t move(const MoveArgs& m, hipStream_t s) {
  const int64_t blocks = (m.entries * LANES + 255) / 256;
  const dim3 grid((unsigned)std::min(blocks, (int64_t)1 << 22));
  if (m.entries * LANES * 32 > (int64_t)64 << 20) evict_move_kernel<LANES, PARAMS, true><<<grid, 256, 0, s>>>(m);
  else evict_move_kernel<LANES, PARAMS, false><<<grid, 256, 0, s>>>(m);
  return hipGetLastError();
}

}  // namespace

size_t evict_workspace(int batch, int heads_kv, int capacity) {
  const int parts = parts_of((int64_t)batch * heads_kv, capacity);
  return parts > 1 ? (size_t)batch * heads_kv * parts * kPartInts * sizeof(int) : 0;
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
  const int64_t pairs = (int64_t)a.batch * a.cache.heads_kv;
  const int capacity = a.cache.table.max_pages * a.cache.table.page.d;
  const PickArgs k = {a, capacity, parts_of(pairs, capacity), (int*)a.workspace};
  if (k.parts > 1) {
    const dim3 grid((unsigned)k.parts, (unsigned)pairs);
    evict_part_kernel<16, 0><<<grid, kThreads, 0, s>>>(k);
    evict_part_kernel<16, 1><<<grid, kThreads, 0, s>>>(k);
    evict_part_kernel<16, 2><<<grid, kThreads, 0, s>>>(k);
    evict_part_kernel<16, 3><<<grid, kThreads, 0, s>>>(k);
  } else if (capacity <= 4 * kThreads) {
    evict_pick_kernel<4><<<(unsigned)pairs, kThreads, 0, s>>>(k);
  } else {
    evict_pick_kernel<16><<<(unsigned)pairs, kThreads, 0, s>>>(k);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int size = a.cache.group ? 1 : a.bf16 ? 2 : 4;
  const PoolView &kc = a.cache.k, &vc = a.cache.v;
  const MoveArgs m = {a, pairs * a.keep, capacity, kc.sp * size, kc.sh * size, kc.ss * size, vc.sp * size, vc.sh * size, vc.ss * size};
  if (!a.cache.group) {
    const int bytes = a.cache.head_dim * size;
    return bytes == 512 ? move<32, 0>(m, s) : bytes == 256 ? move<16, 0>(m, s) : move<8, 0>(m, s);
  }
  if (a.cache.head_dim == 128) return a.cache.group == 32 ? move<4, 4>(m, s) : move<4, 2>(m, s);
  return a.cache.group == 32 ? move<2, 2>(m, s) : move<2, 1>(m, s);
}

}  // namespace seer
