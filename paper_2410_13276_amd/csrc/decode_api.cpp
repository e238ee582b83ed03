// decode_api.cpp -- the C ABI of include/seer_decode.h: validation, then launches on the
// caller's stream.  No memory is owned and no state is kept.
#include "abi_checks.h"

namespace {

seer_status check_paged(const seer_paged_desc* d) {
  if (!d) return SEER_ERR_INVALID_ARG;
  if (d->batch <= 0 || d->heads_q <= 0 || d->heads_kv <= 0 || d->tokens <= 0 || d->reserved != 0)
    return SEER_ERR_INVALID_ARG;
  if (d->heads_q % d->heads_kv != 0 || d->pos_stride < 0) return SEER_ERR_INVALID_ARG;
  seer_status s = check_layout(d->head_dim, d->dtype);
  if (s == SEER_OK) s = check_pages(d->page_size, d->num_pages, d->batch, d->max_pages, d->table_stride);
  if (s == SEER_OK) s = check_strides(d->q_stride, d->dtype);
  if (s == SEER_OK) s = check_written(d->o_stride, {d->batch, d->heads_q, d->tokens}, d->head_dim, d->dtype);
  if (s == SEER_OK) s = check_cache_strides(d->k_cache_stride, d->dtype);
  if (s == SEER_OK) s = check_cache_strides(d->v_cache_stride, d->dtype);
  if (s != SEER_OK) return s;
  const int64_t rows = (int64_t)d->heads_q / d->heads_kv * d->tokens;
  const int64_t blocks = (rows + 15) / 16, items = (int64_t)d->batch * d->heads_kv;
  if (rows > kMostRows || items > kMostRows || items * blocks > kMostRows) return SEER_ERR_UNSUPPORTED;
  return SEER_OK;
}

}  // namespace

extern "C" {

seer_status seer_rope(const seer_rope_desc* d, const seer_rope_params* rope, const void* q, const void* k,
                      void* q_out, void* k_out, const int32_t* positions, int32_t start, int32_t grad,
                      void* stream) {
  if (!d || !rope || !q || !q_out) return SEER_ERR_INVALID_ARG;
  if (d->batch <= 0 || d->heads_q <= 0 || d->heads_kv < 0 || d->seq_len <= 0 || d->pos_stride < 0)
    return SEER_ERR_INVALID_ARG;
  if ((k == nullptr) != (d->heads_kv == 0) || (k_out == nullptr) != (d->heads_kv == 0)) return SEER_ERR_INVALID_ARG;
  seer_status s = check_layout(d->head_dim, d->dtype);
  if (s == SEER_OK) s = check_rope(rope, d->head_dim);
  if (s == SEER_OK) s = check_strides(d->q_stride, d->dtype);
  if (s == SEER_OK) s = check_written(d->q_out_stride, {d->batch, d->heads_q, d->seq_len}, d->head_dim, d->dtype);
  if (s == SEER_OK && d->heads_kv > 0) s = check_strides(d->k_stride, d->dtype);
  if (s == SEER_OK && d->heads_kv > 0)
    s = check_written(d->k_out_stride, {d->batch, d->heads_kv, d->seq_len}, d->head_dim, d->dtype);
  if (s != SEER_OK) return s;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(q_out, 16) || !aligned(k_out, 16) || !aligned(positions, 4))
    return SEER_ERR_INVALID_ARG;
  if ((int64_t)d->batch * d->seq_len > kMostTokens || (int64_t)d->heads_q + d->heads_kv > 65535)
    return SEER_ERR_UNSUPPORTED;
  if (!positions && (int64_t)start + d->seq_len - 1 > INT32_MAX) return SEER_ERR_INVALID_ARG;
  seer::RotateArgs a;
  a.q = view(q, d->q_stride);
  a.k = view(k, d->k_stride);
  a.qo = view(q_out, d->q_out_stride);
  a.ko = view(k_out, d->k_out_stride);
  a.batch = d->batch;
  a.heads_q = d->heads_q;
  a.heads_kv = d->heads_kv;
  a.seq_len = d->seq_len;
  a.head_dim = d->head_dim;
  a.bf16 = d->dtype == SEER_BF16;
  a.grad = grad != 0;
  a.rope = rope_view(rope);
  a.positions = positions;
  a.pos_stride = d->pos_stride;
  a.start = start;
  return from_hip(seer::launch_rotate(a, static_cast<hipStream_t>(stream)));
}

seer_status seer_kv_append(const seer_append_desc* d, const seer_rope_params* rope, const void* k, const void* v,
                           void* k_cache, void* v_cache, const int32_t* table, const int32_t* positions,
                           const int32_t* rows, void* stream) {
  if (!d || !k || !v || !k_cache || !v_cache || !table || !positions) return SEER_ERR_INVALID_ARG;
  if (d->batch <= 0 || d->tokens <= 0 || d->heads_kv <= 0 || d->pos_stride < 0 || d->reserved != 0)
    return SEER_ERR_INVALID_ARG;
  seer_status s = check_layout(d->head_dim, d->dtype);
  if (s == SEER_OK && rope) s = check_rope(rope, d->head_dim);
  if (s == SEER_OK) s = check_pages(d->page_size, d->num_pages, d->table_rows, d->max_pages, d->table_stride);
  if (s == SEER_OK) s = check_strides(d->k_stride, d->dtype);
  if (s == SEER_OK) s = check_strides(d->v_stride, d->dtype);
  const int32_t places[3] = {d->num_pages, d->heads_kv, d->page_size};
  if (s == SEER_OK) s = check_written(d->k_cache_stride, places, d->head_dim, d->dtype);
  if (s == SEER_OK) s = check_written(d->v_cache_stride, places, d->head_dim, d->dtype);
  if (s != SEER_OK) return s;
  if (!rows && d->table_rows < d->batch) return SEER_ERR_INVALID_ARG;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(table, 4) ||
      !aligned(positions, 4) || !aligned(rows, 4))
    return SEER_ERR_INVALID_ARG;
  if ((int64_t)d->batch * d->tokens > kMostTokens || d->heads_kv > 65535) return SEER_ERR_UNSUPPORTED;
  seer::AppendArgs a;
  a.k = view(k, d->k_stride);
  a.v = view(v, d->v_stride);
  a.kc = cache(k_cache, d->k_cache_stride);
  a.vc = cache(v_cache, d->v_cache_stride);
  a.table = table_view(table, d->table_stride, d->table_rows, d->max_pages, d->num_pages, d->page_size);
  a.batch = d->batch;
  a.tokens = d->tokens;
  a.heads_kv = d->heads_kv;
  a.head_dim = d->head_dim;
  a.bf16 = d->dtype == SEER_BF16;
  a.rope = rope_view(rope);
  a.positions = positions;
  a.rows = rows;
  a.pos_stride = d->pos_stride;
  return from_hip(seer::launch_append(a, static_cast<hipStream_t>(stream)));
}

size_t seer_paged_attn_workspace_bytes(const seer_paged_desc* d) {
  if (check_paged(d) != SEER_OK) return 0;
  return seer::paged_attn_workspace(d->batch, d->heads_q, d->heads_kv, d->tokens, d->head_dim);
}

seer_status seer_paged_attn(const seer_paged_desc* d, const seer_rope_params* rope, float sm_scale, const void* q,
                            const void* k_cache, const void* v_cache, const int32_t* table,
                            const int32_t* positions, void* o, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream) {
  seer_status s = check_paged(d);
  if (s == SEER_OK && rope) s = check_rope(rope, d->head_dim);
  if (s != SEER_OK) return s;
  if (!q || !k_cache || !v_cache || !table || !positions || !o) return SEER_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(o, 16) || !aligned(lse, 4) ||
      !aligned(table, 4) || !aligned(positions, 4))
    return SEER_ERR_INVALID_ARG;
  if (!std::isfinite(sm_scale)) return SEER_ERR_INVALID_ARG;
  // (the weights are powers of 2, and an infinite sm_scale log2(e) would make the largest one 2^(0 inf))
  if (sm_scale > 0x1p127f) return SEER_ERR_INVALID_ARG;
  if (!workspace ||
      workspace_bytes < seer::paged_attn_workspace(d->batch, d->heads_q, d->heads_kv, d->tokens, d->head_dim))
    return SEER_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return SEER_ERR_INVALID_ARG;
  seer::PagedArgs a;
  a.q = view(q, d->q_stride);
  a.o = o;
  a.osb = d->o_stride[0];
  a.osh = d->o_stride[1];
  a.oss = d->o_stride[2];
  a.lse = lse;
  a.kc = cache(k_cache, d->k_cache_stride);
  a.vc = cache(v_cache, d->v_cache_stride);
  a.table = table_view(table, d->table_stride, d->batch, d->max_pages, d->num_pages, d->page_size);
  a.positions = positions;
  a.pos_stride = d->pos_stride;
  a.batch = d->batch;
  a.heads_q = d->heads_q;
  a.heads_kv = d->heads_kv;
  a.tokens = d->tokens;
  a.head_dim = d->head_dim;
  a.bf16 = d->dtype == SEER_BF16;
  a.rope = rope_view(rope);
  a.scale = sm_scale > 0.f ? sm_scale : (float)(1.0 / std::sqrt((double)d->head_dim));
  a.workspace = workspace;
  return from_hip(seer::launch_paged_attn(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
