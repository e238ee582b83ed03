// cache.h -- internal launchers behind include/seer_cache.h.  Arguments are validated by the ABI layer.
#pragma once

#include "decode.h"

namespace seer {

struct PoolView {
  const void* data;
  const uint32_t* params;  // (step, middle) pairs, the step in the low half
  int64_t sp, sh, ss;      // strides of data: elements, or bytes of codes
  int64_t psp, psh, pss;   // of params: pairs
};

struct CacheArgs {
  PoolView k, v;
  PageTable table;
  int heads_kv, head_dim, group;  // group 0: values of the call's type
};

struct StoreArgs {  // append (k, v read) and read (k, v written)
  CacheArgs cache;
  TensorView k, v;
  int batch, tokens;
  bool bf16;
  RopeView rope;
  const int32_t* positions;
  const int32_t* rope_positions;
  const int32_t* rows;
  int64_t pos_stride;
};

struct QueryArgs {
  CacheArgs cache;
  TensorView q;
  int batch, heads_q, tokens;
  bool bf16;
  RopeView rope;
  const int32_t* positions;
  const int32_t* rope_positions;  // (positions where the call has none)
  int64_t pos_stride;
  float scale;
};

struct Q4AttnArgs {
  QueryArgs q;
  void* o;
  int64_t osb, osh, oss;
  float* lse;
  void* workspace;
};

struct WeightArgs {
  QueryArgs q;
  const float* lse;
  const float* in;
  float* out;
  int64_t isb, ish, osb, osh;
  int width;
  float decay;
};

struct EvictArgs {
  CacheArgs cache;
  int batch, keep, first, last;
  bool bf16;  // of a cache of group 0
  const int32_t* lengths;
  int32_t* new_lengths;
  PageTable to;
  const float* weights;
  float* new_weights;
  int width, new_width;
  int64_t sb, sh, nsb, nsh;
  int32_t* kept;
  void* workspace;
};

hipError_t launch_append_q4(const StoreArgs& a, hipStream_t s);
hipError_t launch_read(const StoreArgs& a, hipStream_t s);
hipError_t launch_q4_attn(const Q4AttnArgs& a, hipStream_t s);
size_t q4_attn_workspace(int batch, int heads_q, int heads_kv, int tokens, int head_dim, int group);
hipError_t launch_weights(const WeightArgs& a, hipStream_t s);
hipError_t launch_evict(const EvictArgs& a, hipStream_t s);
size_t evict_workspace(int batch, int heads_kv, int capacity);

}  // namespace seer
