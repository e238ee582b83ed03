// abi_checks.h -- what the parts of the C ABI share in checking and passing on their arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "decode.h"
#include "seer_decode.h"

namespace {

constexpr int64_t kMostTokens = (int64_t)1 << 27;    // of one rope or append call (a launch holds less than 2^32 threads)
constexpr int64_t kMostKeys = (int64_t)1 << 30;      // of one table row
constexpr int64_t kMostRows = (int64_t)1 << 23;      // query rows of one KV head, and blocks of 16 of them, of one attention call

[[maybe_unused]] bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Head dimension, type and the strides of some [..][..][rows][head_dim] tensors.
[[maybe_unused]] seer_status check_layout(int32_t head_dim, int32_t dtype) {
  if (dtype != SEER_BF16 && dtype != SEER_F32) return SEER_ERR_INVALID_ARG;
  if (head_dim <= 0) return SEER_ERR_INVALID_ARG;
  return head_dim == 64 || head_dim == 128 ? SEER_OK : SEER_ERR_UNSUPPORTED;
}
[[maybe_unused]] seer_status check_strides(const int64_t (&st)[3], int32_t dtype) {
  const int64_t vec = dtype == SEER_F32 ? 4 : 8;  // elements of a 16-byte access
  for (int64_t x : st)
    if (x < 0 || x % vec != 0) return SEER_ERR_UNSUPPORTED;
  return SEER_OK;
}

// A buffer that is written: no two heads or tokens at the same place.
[[maybe_unused]] seer_status check_written(const int64_t (&st)[3], const int32_t (&n)[3], int32_t head_dim, int32_t dtype) {
  const seer_status s = check_strides(st, dtype);
  if (s != SEER_OK) return s;
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1 && st[i] < head_dim) return SEER_ERR_INVALID_ARG;
  return SEER_OK;
}

// The attention counts a cache's strides in 16-byte pieces of 32 bits.
[[maybe_unused]] seer_status check_cache_strides(const int64_t (&st)[3], int32_t dtype) {
  const seer_status s = check_strides(st, dtype);
  if (s != SEER_OK) return s;
  const int64_t vec = dtype == SEER_F32 ? 4 : 8;
  return st[0] / vec <= UINT32_MAX && st[2] / vec <= UINT32_MAX ? SEER_OK : SEER_ERR_UNSUPPORTED;
}

[[maybe_unused]] seer_status check_rope(const seer_rope_params* r, int32_t head_dim) {
  if (!r->inv_freq || !aligned(r->inv_freq, 8)) return SEER_ERR_INVALID_ARG;
  if (r->rot_dim <= 0 || r->rot_dim > head_dim) return SEER_ERR_INVALID_ARG;
  if (r->rot_dim % 16 != 0) return SEER_ERR_UNSUPPORTED;
  if (r->interleaved != 0 && r->interleaved != 1) return SEER_ERR_INVALID_ARG;
  return std::isfinite(r->scale) ? SEER_OK : SEER_ERR_INVALID_ARG;
}

[[maybe_unused]] seer_status check_pages(int32_t page_size, int32_t num_pages, int32_t rows, int32_t max_pages, int64_t table_stride) {
  if (page_size <= 0 || num_pages <= 0 || rows <= 0 || max_pages <= 0) return SEER_ERR_INVALID_ARG;
  if (table_stride < 0) return SEER_ERR_INVALID_ARG;
  return (int64_t)page_size * max_pages <= kMostKeys ? SEER_OK : SEER_ERR_UNSUPPORTED;
}

[[maybe_unused]] seer::TensorView view(const void* p, const int64_t (&st)[3]) { return {p, st[0], st[1], st[2]}; }
[[maybe_unused]] seer::CacheView cache(const void* p, const int64_t (&st)[3]) { return {p, st[0], st[1], st[2]}; }

[[maybe_unused]] seer::RopeView rope_view(const seer_rope_params* r) {
  if (!r) return {nullptr, 0, 0, 1.f};
  return {r->inv_freq, r->rot_dim, r->interleaved, r->scale};
}

[[maybe_unused]] seer::PageTable table_view(const int32_t* t, int64_t stride, int rows, int max_pages, int num_pages, int page_size) {
  return {t, stride, rows, max_pages, num_pages, seer::fast_div(page_size)};
}

[[maybe_unused]] seer_status from_hip(hipError_t e) { return e == hipSuccess ? SEER_OK : SEER_ERR_HIP; }

}  // namespace
