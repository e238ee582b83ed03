// cache_api.cpp -- the C ABI of include/seer_cache.h: validation, then launches on the caller's stream.
// No memory is owned and no state is kept.
#include "abi_checks.h"
#include "cache.h"
#include "seer_cache.h"

namespace {

constexpr int64_t kMostPairs = ((int64_t)1 << 22) - 1;  // of sequence and KV head, of one eviction (workgroups of 1024, less than 2^32 threads)
constexpr float kMostScale = 0x1p100f;            // (16 log2(e) times it is finite, which the weights' arguments need)

// One pool's pointers and strides.
seer_status check_pool(const seer_kv_cache* c, const seer_kv_pool& p, bool written) {
  if (!p.data || !aligned(p.data, 16)) return SEER_ERR_INVALID_ARG;
  const int64_t vec = c->group ? 16 : c->dtype == SEER_F32 ? 4 : 8;  // elements of 16 bytes
  const int64_t size = c->group ? c->head_dim / 2 : c->head_dim;
  const int64_t places[3] = {c->num_pages, c->heads_kv, c->page_size};
  for (int i = 0; i < 3; ++i) {
    if (p.stride[i] < 0 || p.stride[i] % vec != 0) return SEER_ERR_UNSUPPORTED;
    if (written && places[i] > 1 && p.stride[i] < size) return SEER_ERR_INVALID_ARG;
  }
  if (!c->group) return SEER_OK;
  const int64_t groups = c->head_dim / c->group;
  if (!p.params || !aligned(p.params, 4 * groups)) return SEER_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i) {
    if (p.param_stride[i] < 0 || p.param_stride[i] % groups != 0) return SEER_ERR_UNSUPPORTED;
    if (written && places[i] > 1 && p.param_stride[i] < groups) return SEER_ERR_INVALID_ARG;
  }
  return SEER_OK;
}

seer_status check_cache(const seer_kv_cache* c, bool values, bool written) {
  if (!c || c->heads_kv <= 0) return SEER_ERR_INVALID_ARG;
  if (c->group != 0 && c->group != 32 && c->group != 64) return SEER_ERR_UNSUPPORTED;
  seer_status s = check_layout(c->head_dim, c->group ? (int32_t)SEER_BF16 : c->dtype);
  if (s == SEER_OK) s = check_pages(c->page_size, c->num_pages, c->table_rows, c->max_pages, c->table_stride);
  if (s != SEER_OK) return s;
  if (!c->table || !aligned(c->table, 4)) return SEER_ERR_INVALID_ARG;
  s = check_pool(c, c->k, written);
  if (s == SEER_OK && values) s = check_pool(c, c->v, written);
  if (s != SEER_OK) return s;
  return c->heads_kv <= 65535 ? SEER_OK : SEER_ERR_UNSUPPORTED;
}

// Tokens that are stored, or (written) read.
seer_status check_tokens(const seer_kv_cache* c, const seer_kv_tokens* d, const void* k, const void* v,
                         const int32_t* positions, const int32_t* rows, bool written) {
  if (!d || !k || !v || !positions) return SEER_ERR_INVALID_ARG;
  if (d->batch <= 0 || d->tokens <= 0 || d->pos_stride < 0 || d->reserved != 0) return SEER_ERR_INVALID_ARG;
  seer_status s = check_layout(c->head_dim, d->dtype);
  const int32_t n[3] = {d->batch, c->heads_kv, d->tokens};
  if (s == SEER_OK) s = written ? check_written(d->k_stride, n, c->head_dim, d->dtype) : check_strides(d->k_stride, d->dtype);
  if (s == SEER_OK) s = written ? check_written(d->v_stride, n, c->head_dim, d->dtype) : check_strides(d->v_stride, d->dtype);
  if (s != SEER_OK) return s;
  if (!rows && c->table_rows < d->batch) return SEER_ERR_INVALID_ARG;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(positions, 4) || !aligned(rows, 4)) return SEER_ERR_INVALID_ARG;
  return (int64_t)d->batch * d->tokens <= kMostTokens ? SEER_OK : SEER_ERR_UNSUPPORTED;
}

seer_status check_queries(const seer_kv_cache* c, const seer_kv_queries* d) {
  if (!d || d->batch <= 0 || d->heads_q <= 0 || d->tokens <= 0 || d->pos_stride < 0) return SEER_ERR_INVALID_ARG;
  if (d->heads_q % c->heads_kv != 0 || c->table_rows < d->batch) return SEER_ERR_INVALID_ARG;
  seer_status s = check_layout(c->head_dim, d->dtype);
  if (s == SEER_OK) s = check_strides(d->q_stride, d->dtype);
  if (s != SEER_OK) return s;
  const int64_t rows = (int64_t)d->heads_q / c->heads_kv * d->tokens;
  const int64_t blocks = (rows + 15) / 16, items = (int64_t)d->batch * c->heads_kv;
  if (rows > kMostRows || items > kMostRows || items * blocks > kMostRows) return SEER_ERR_UNSUPPORTED;
  return SEER_OK;
}

seer_status check_scale(float sm_scale) {
  return std::isfinite(sm_scale) && sm_scale <= kMostScale ? SEER_OK : SEER_ERR_INVALID_ARG;
}

seer::CacheArgs cache_args(const seer_kv_cache* c) {
  auto pool = [](const seer_kv_pool& p) -> seer::PoolView {
    return {p.data, static_cast<const uint32_t*>(p.params), p.stride[0], p.stride[1], p.stride[2],
            p.param_stride[0], p.param_stride[1], p.param_stride[2]};
  };
  return {pool(c->k), pool(c->v), table_view(c->table, c->table_stride, c->table_rows, c->max_pages, c->num_pages, c->page_size),
          c->heads_kv, c->head_dim, c->group};
}

seer::StoreArgs store_args(const seer_kv_cache* c, const seer_kv_tokens* d, const seer_rope_params* rope, const void* k,
                           const void* v, const int32_t* positions, const int32_t* rope_positions, const int32_t* rows) {
  return {cache_args(c), view(k, d->k_stride), view(v, d->v_stride), d->batch, d->tokens, d->dtype == SEER_BF16, rope_view(rope),
          positions, rope_positions ? rope_positions : positions, rows, d->pos_stride};
}

seer::QueryArgs query_args(const seer_kv_cache* c, const seer_kv_queries* d, const seer_rope_params* rope, float sm_scale,
                           const void* q, const int32_t* positions, const int32_t* rope_positions) {
  return {cache_args(c), view(q, d->q_stride), d->batch, d->heads_q, d->tokens, d->dtype == SEER_BF16, rope_view(rope),
          positions, rope_positions ? rope_positions : positions, d->pos_stride,
          sm_scale > 0.f ? sm_scale : (float)(1.0 / std::sqrt((double)c->head_dim))};
}

// The attention counts page and slot strides in rows of 16 bytes, and of params, in 32 bits.
seer_status check_near(const seer_kv_cache* c, const seer_kv_pool& p) {
  for (int i = 0; i < 3; i += 2)
    if (p.stride[i] / 16 > UINT32_MAX || p.param_stride[i] / (c->head_dim / c->group) > UINT32_MAX) return SEER_ERR_UNSUPPORTED;
  return SEER_OK;
}

seer_status check_attn(const seer_kv_cache* c, const seer_kv_queries* d) {
  seer_status s = check_cache(c, true, false);
  if (s == SEER_OK && c->group == 0) s = SEER_ERR_INVALID_ARG;
  if (s == SEER_OK) s = check_near(c, c->k);
  if (s == SEER_OK) s = check_near(c, c->v);
  if (s == SEER_OK) s = check_queries(c, d);
  if (s == SEER_OK) s = check_written(d->o_stride, {d->batch, d->heads_q, d->tokens}, c->head_dim, d->dtype);
  return s;
}

size_t attn_workspace(const seer_kv_cache* c, const seer_kv_queries* d) {
  return seer::q4_attn_workspace(d->batch, d->heads_q, c->heads_kv, d->tokens, c->head_dim, c->group);
}

}  // namespace

extern "C" {

seer_status seer_kv_append_q4(const seer_kv_cache* c, const seer_kv_tokens* d, const seer_rope_params* rope,
                              const void* k, const void* v, const int32_t* positions, const int32_t* rope_positions,
                              const int32_t* rows, void* stream) {
  seer_status s = check_cache(c, true, true);
  if (s == SEER_OK && c->group == 0) s = SEER_ERR_INVALID_ARG;
  if (s == SEER_OK) s = check_tokens(c, d, k, v, positions, rows, false);
  if (s == SEER_OK && rope) s = check_rope(rope, c->head_dim);
  if (s == SEER_OK && !aligned(rope_positions, 4)) s = SEER_ERR_INVALID_ARG;
  if (s != SEER_OK) return s;
  return from_hip(seer::launch_append_q4(store_args(c, d, rope, k, v, positions, rope_positions, rows),
                                         static_cast<hipStream_t>(stream)));
}

seer_status seer_kv_read(const seer_kv_cache* c, const seer_kv_tokens* d, void* k, void* v, const int32_t* positions,
                         const int32_t* rows, void* stream) {
  seer_status s = check_cache(c, true, false);
  if (s == SEER_OK) s = check_tokens(c, d, k, v, positions, rows, true);
  if (s == SEER_OK && c->group == 0 && d->dtype != c->dtype) s = SEER_ERR_INVALID_ARG;
  if (s != SEER_OK) return s;
  return from_hip(seer::launch_read(store_args(c, d, nullptr, k, v, positions, nullptr, rows), static_cast<hipStream_t>(stream)));
}

size_t seer_paged_attn_q4_workspace_bytes(const seer_kv_cache* c, const seer_kv_queries* d) {
  return check_attn(c, d) == SEER_OK ? attn_workspace(c, d) : 0;
}

seer_status seer_paged_attn_q4(const seer_kv_cache* c, const seer_kv_queries* d, const seer_rope_params* rope,
                               float sm_scale, const void* q, const int32_t* positions, const int32_t* rope_positions,
                               void* o, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  seer_status s = check_attn(c, d);
  if (s == SEER_OK && rope) s = check_rope(rope, c->head_dim);
  if (s == SEER_OK) s = check_scale(sm_scale);
  if (s != SEER_OK) return s;
  if (!q || !positions || !o) return SEER_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(o, 16) || !aligned(lse, 4) || !aligned(positions, 4) || !aligned(rope_positions, 4))
    return SEER_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < attn_workspace(c, d)) return SEER_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return SEER_ERR_INVALID_ARG;
  return from_hip(seer::launch_q4_attn({query_args(c, d, rope, sm_scale, q, positions, rope_positions), o, d->o_stride[0],
                                        d->o_stride[1], d->o_stride[2], lse, workspace}, static_cast<hipStream_t>(stream)));
}

seer_status seer_kv_weights(const seer_kv_cache* c, const seer_kv_queries* d, const seer_rope_params* rope,
                            float sm_scale, const void* q, const int32_t* positions, const int32_t* rope_positions,
                            const float* lse, const seer_kv_weight_buf* w, void* stream) {
  seer_status s = check_cache(c, false, false);
  if (s == SEER_OK) s = check_queries(c, d);
  if (s == SEER_OK && c->group == 0 && d->dtype != c->dtype) s = SEER_ERR_INVALID_ARG;
  if (s == SEER_OK && rope) s = check_rope(rope, c->head_dim);
  if (s == SEER_OK) s = check_scale(sm_scale);
  if (s != SEER_OK) return s;
  if (!q || !positions || !lse || !w || !w->out || w->width <= 0 || !std::isfinite(w->decay)) return SEER_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(lse, 4) || !aligned(positions, 4) || !aligned(rope_positions, 4) || !aligned(w->in, 4) ||
      !aligned(w->out, 4))
    return SEER_ERR_INVALID_ARG;
  if (w->decay != 0.f && !w->in) return SEER_ERR_INVALID_ARG;
  const int32_t n[2] = {d->batch, c->heads_kv};
  for (int i = 0; i < 2; ++i) {
    if (w->in_stride[i] < 0 || w->out_stride[i] < 0) return SEER_ERR_INVALID_ARG;
    if (n[i] > 1 && w->out_stride[i] < w->width) return SEER_ERR_INVALID_ARG;
    if (n[i] > 1 && w->decay != 0.f && w->in == w->out && w->in_stride[i] != w->out_stride[i]) return SEER_ERR_INVALID_ARG;
  }
  return from_hip(seer::launch_weights({query_args(c, d, rope, sm_scale, q, positions, rope_positions), lse, w->in, w->out,
                                        w->in_stride[0], w->in_stride[1], w->out_stride[0], w->out_stride[1], w->width, w->decay},
                                       static_cast<hipStream_t>(stream)));
}

size_t seer_kv_evict_workspace_bytes(const seer_kv_cache* c, int32_t batch) {
  if (check_cache(c, false, false) != SEER_OK || batch <= 0 || (int64_t)batch * c->heads_kv > kMostPairs) return 0;
  return seer::evict_workspace(batch, c->heads_kv, c->page_size * c->max_pages);
}

seer_status seer_kv_evict(const seer_kv_cache* c, const seer_kv_eviction* d, void* workspace, size_t workspace_bytes,
                          void* stream) {
  seer_status s = check_cache(c, true, true);
  if (s != SEER_OK) return s;
  if (!d || d->batch <= 0 || d->keep <= 0 || d->first < 0 || d->last < 0 || d->width <= 0 || d->reserved != 0)
    return SEER_ERR_INVALID_ARG;
  if ((int64_t)d->first + d->last > d->keep || d->new_width < d->keep || c->table_rows < d->batch) return SEER_ERR_INVALID_ARG;
  if (!d->lengths || !d->new_lengths || !d->new_table || !d->weights || !d->new_weights || !d->kept) return SEER_ERR_INVALID_ARG;
  if (!aligned(d->lengths, 4) || !aligned(d->new_lengths, 4) || !aligned(d->new_table, 4) || !aligned(d->weights, 4) ||
      !aligned(d->new_weights, 4) || !aligned(d->kept, 4))
    return SEER_ERR_INVALID_ARG;
  s = check_pages(c->page_size, c->num_pages, d->batch, d->new_max_pages, d->new_table_stride);
  if (s != SEER_OK) return s;
  if ((int64_t)c->page_size * d->new_max_pages < d->keep || d->weights == d->new_weights) return SEER_ERR_INVALID_ARG;
  const int32_t n[2] = {d->batch, c->heads_kv};
  for (int i = 0; i < 2; ++i) {
    if (d->stride[i] < 0 || d->new_stride[i] < 0) return SEER_ERR_INVALID_ARG;
    if (n[i] > 1 && d->new_stride[i] < d->new_width) return SEER_ERR_INVALID_ARG;
  }
  if ((int64_t)d->batch * c->heads_kv > kMostPairs) return SEER_ERR_UNSUPPORTED;
  const size_t need = seer::evict_workspace(d->batch, c->heads_kv, c->page_size * c->max_pages);
  if (need && (!workspace || workspace_bytes < need)) return SEER_ERR_WORKSPACE;
  if (need && !aligned(workspace, 256)) return SEER_ERR_INVALID_ARG;
  seer::EvictArgs a;
  a.cache = cache_args(c);
  a.batch = d->batch;
  a.keep = d->keep;
  a.first = d->first;
  a.last = d->last;
  a.bf16 = c->dtype == SEER_BF16;
  a.lengths = d->lengths;
  a.new_lengths = d->new_lengths;
  a.to = table_view(d->new_table, d->new_table_stride, d->batch, d->new_max_pages, c->num_pages, c->page_size);
  a.weights = d->weights;
  a.new_weights = d->new_weights;
  a.width = d->width;
  a.new_width = d->new_width;
  a.sb = d->stride[0];
  a.sh = d->stride[1];
  a.nsb = d->new_stride[0];
  a.nsh = d->new_stride[1];
  a.kept = d->kept;
  a.workspace = workspace;
  return from_hip(seer::launch_evict(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
