// What the C-ABI entry points share on the host: the error text and the checks
// of tensor descriptors.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
#include <mutex>
#include <string>

#include "../../include/mla_sparse.h"

namespace mla {
namespace host {

inline thread_local std::string g_last_error;

inline mla_status_t fail(mla_status_t st, const std::string& msg) {
  g_last_error = msg;
  return st;
}

struct Extent {
  uintptr_t lo, hi;  // [lo, hi) bytes touched
};

inline int dtype_size(int32_t dt) {
  switch (dt) {
    case MLA_DTYPE_BF16: return 2;
    case MLA_DTYPE_FP8_E4M3FN: return 1;
    case MLA_DTYPE_MXFP4: return 1;
    case MLA_DTYPE_FP32: return 4;
    case MLA_DTYPE_INT32: return 4;
    default: return 0;
  }
}

inline int64_t numel(const mla_tensor_t& t) {
  int64_t n = 1;
  for (int d = 0; d < t.ndim; ++d) n *= t.shape[d];
  return n;
}

inline Extent extent(const mla_tensor_t& t) {
  const int es = dtype_size(t.dtype);
  if (numel(t) == 0) return {0, 0};
  int64_t hi = 0;
  for (int d = 0; d < t.ndim; ++d) hi += (t.shape[d] - 1) * t.stride[d];
  const uintptr_t base = reinterpret_cast<uintptr_t>(t.data);
  return {base, base + (uintptr_t)((hi + 1) * es)};
}

inline bool overlaps(const Extent& a, const Extent& b) {
  if (a.lo == a.hi || b.lo == b.hi) return false;
  return a.lo < b.hi && b.lo < a.hi;
}

// Common checks of one descriptor.  `name` is used in messages.
inline mla_status_t check_tensor(const mla_tensor_t* t, const char* name, int32_t dtype, int ndim,
                          bool allow_scale = false) {
  if (!t) return fail(MLA_ERR_INVALID_ARGUMENT, std::string(name) + ": null descriptor");
  if (t->dtype != dtype)
    return fail(MLA_ERR_INVALID_ARGUMENT, std::string(name) + ": wrong dtype " + std::to_string(t->dtype));
  if (t->ndim != ndim)
    return fail(MLA_ERR_INVALID_ARGUMENT, std::string(name) + ": expected " + std::to_string(ndim) +
                                              " dims, got " + std::to_string(t->ndim));
  for (int d = 0; d < ndim; ++d)
    if (t->shape[d] < 0 || t->stride[d] < 0)
      return fail(MLA_ERR_INVALID_ARGUMENT, std::string(name) + ": negative shape or stride");
  // (a tensor of no elements has no strides to speak of)
  if (ndim > 0 && t->shape[ndim - 1] > 1 && t->stride[ndim - 1] != 1 && numel(*t) > 0)
    return fail(MLA_ERR_INVALID_ARGUMENT, std::string(name) + ": innermost stride must be 1");
  if (numel(*t) > 0 && !t->data)
    return fail(MLA_ERR_INVALID_ARGUMENT, std::string(name) + ": null data pointer");
  if (!allow_scale && t->block_scale)
    return fail(MLA_ERR_INVALID_ARGUMENT, std::string(name) + ": block_scale must be NULL");
  return MLA_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Row-major contiguous with the given shape.
inline bool contiguous(const mla_tensor_t& t, std::initializer_list<int64_t> shape) {
  if (t.ndim != (int)shape.size()) return false;
  int d = 0;
  for (int64_t v : shape)
    if (t.shape[d++] != v) return false;
  int64_t st = 1;
  if (numel(t) == 0) return true;
  for (int k = t.ndim - 1; k >= 0; --k) {
    if (t.shape[k] > 1 && t.stride[k] != st) return false;
    st *= t.shape[k];
  }
  return true;
}

// Rows of a [.., .., .., D] tensor are 16-byte aligned: base and every outer stride.
inline bool rows_aligned(const mla_tensor_t& t, int es) {
  if (!aligned16(t.data)) return false;
  for (int d = 0; d + 1 < t.ndim; ++d)
    if ((t.stride[d] * es) % 16 != 0) return false;
  return true;
}

// No element of the tensor shares its place with another (an output's rows).
inline bool rows_apart(const mla_tensor_t& t) {
  if (numel(t) == 0) return true;
  bool done[4] = {};
  int64_t hi = 0;  // the last element of the dims taken so far, smallest stride first
  for (int k = 0; k < t.ndim; ++k) {
    int d = -1;
    for (int e = 0; e < t.ndim; ++e)
      if (!done[e] && (d < 0 || t.stride[e] < t.stride[d])) d = e;
    done[d] = true;
    if (t.shape[d] == 1) continue;
    if (t.stride[d] <= hi) return false;
    hi += (t.shape[d] - 1) * t.stride[d];
  }
  return true;
}

// The split-K workspace of a stream, at least `bytes` of it (mla_api.hip); the caller
// keeps `lock` until the kernels that use it are queued.
mla_status_t get_workspace(hipStream_t stream, size_t bytes, void** out, std::unique_lock<std::mutex>& lock);
int device_cus();

inline bool shape_is(const mla_tensor_t* t, std::initializer_list<int64_t> s) {
  int d = 0;
  for (int64_t v : s)
    if (t->shape[d++] != v) return false;
  return true;
}

// The pools of an attention call: types, shapes, then layout.  The latent pool is
// bf16, e4m3 (the RoPE pool alike, both with scales) or 4 bits (the RoPE pool bf16).
inline mla_status_t check_pool_types(const mla_tensor_t* ckv_pool, const mla_tensor_t* kpe_pool) {
  const int32_t kv_dtype = ckv_pool->dtype;
  if (kv_dtype != MLA_DTYPE_BF16 && kv_dtype != MLA_DTYPE_FP8_E4M3FN && kv_dtype != MLA_DTYPE_MXFP4)
    return fail(MLA_ERR_INVALID_ARGUMENT, "ckv_pool: dtype must be bf16 or fp8-e4m3fn or mxfp4");
  const bool fp8 = kv_dtype == MLA_DTYPE_FP8_E4M3FN;
  mla_status_t st;
  if ((st = check_tensor(ckv_pool, "ckv_pool", kv_dtype, 3, fp8)) != MLA_OK) return st;
  const int32_t pe_dtype = kv_dtype == MLA_DTYPE_MXFP4 ? (int32_t)MLA_DTYPE_BF16 : kv_dtype;
  if ((st = check_tensor(kpe_pool, "kpe_pool", pe_dtype, 3, fp8)) != MLA_OK) return st;
  if (fp8 && (!ckv_pool->block_scale || !kpe_pool->block_scale))
    return fail(MLA_ERR_INVALID_ARGUMENT, "fp8 pools need block_scale");
  return MLA_OK;
}

inline int64_t latent_row(const mla_tensor_t& ckv_pool) { return ckv_pool.dtype == MLA_DTYPE_MXFP4 ? MLA_MX4_ROW : MLA_DLAT; }

inline mla_status_t check_pool_shapes(const mla_tensor_t& ckv_pool, const mla_tensor_t& kpe_pool) {
  const int64_t P = ckv_pool.shape[0];
  if (!shape_is(&ckv_pool, {P, MLA_BLOCK, latent_row(ckv_pool)}))
    return fail(MLA_ERR_INVALID_ARGUMENT, "ckv_pool: shape must be [P, 64, 512] (MXFP4: [P, 64, 272])");
  if (!shape_is(&kpe_pool, {P, MLA_BLOCK, MLA_DPE}))
    return fail(MLA_ERR_INVALID_ARGUMENT, "kpe_pool: shape must be [P, 64, 64] with the P of ckv_pool");
  return MLA_OK;
}

inline mla_status_t check_pool_layout(const mla_tensor_t& ckv_pool, const mla_tensor_t& kpe_pool) {
  const int64_t row = latent_row(ckv_pool);
  if (ckv_pool.stride[0] != MLA_BLOCK * row || ckv_pool.stride[1] != row ||
      kpe_pool.stride[0] != MLA_BLOCK * MLA_DPE || kpe_pool.stride[1] != MLA_DPE)
    return fail(MLA_ERR_INVALID_ARGUMENT, "pools must be contiguous");
  if (!aligned16(ckv_pool.data) || !aligned16(kpe_pool.data))
    return fail(MLA_ERR_INVALID_ARGUMENT, "pools must be 16-byte aligned");
  return MLA_OK;
}

}  // namespace host
}  // namespace mla
