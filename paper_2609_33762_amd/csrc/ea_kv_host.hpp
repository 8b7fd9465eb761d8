// What the entry points of the cache operators share: checks of arguments, the
// device of a call.
#pragma once

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cstdint>

#include "ea.h"
#include "ea_internal.hpp"
#include "ea_kv_ops.hpp"

namespace ea {
const ea_cache_desc &cache_desc(const ea_cache *c);
int cache_device(const ea_cache *c);
}  // namespace ea

#define KV_HIP(expr)               \
  do {                             \
    hipError_t e_ = (expr);        \
    if (e_ != hipSuccess) {        \
      ea::set_last_hip((int)e_);   \
      return EA_EHIP;              \
    }                              \
  } while (0)

#define KV_TRY(expr)              \
  do {                            \
    int rc_ = (expr);             \
    if (rc_ != EA_OK) return rc_; \
  } while (0)

namespace ea::host {

// The cache's device is current for the duration of a call.
class OnDevice {
 public:
  explicit OnDevice(int dev) {
    if (hipGetDevice(&prev_) != hipSuccess) prev_ = -1;
    if (prev_ != dev) {
      err_ = hipSetDevice(dev);
      changed_ = err_ == hipSuccess;
    }
  }
  ~OnDevice() {
    if (changed_ && prev_ >= 0) (void)hipSetDevice(prev_);
  }
  hipError_t status() const { return err_; }

 private:
  int prev_ = -1;
  bool changed_ = false;
  hipError_t err_ = hipSuccess;
};

inline bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

inline int check_batch(const ea_cache_desc &d, const ea_batch *b) {
  if (!b || b->n_seqs < 0 || b->n_rows < 0 || b->max_rows < 0 || b->max_kv < 0 ||
      b->table_stride < 0)
    return EA_EINVAL;
  if (b->n_seqs == 0 || b->n_rows == 0 || b->max_rows == 0) return EA_OK;
  if (!b->kv_len || !aligned(b->kv_len, 4) || (b->row_start && !aligned(b->row_start, 4)))
    return EA_EINVAL;
  if (!b->page_table || !aligned(b->page_table, 4)) return EA_EINVAL;
  if (b->max_kv > (1 << 30) || b->max_kv < 1) return EA_EINVAL;
  if (b->table_stride > INT32_MAX ||
      b->table_stride < ((int64_t)b->max_kv + d.page_tokens - 1) / d.page_tokens)
    return EA_EINVAL;
  if (!b->row_start && (b->max_rows != 1 || b->n_rows != b->n_seqs)) return EA_EINVAL;
  if (b->max_rows > b->n_rows) return EA_EINVAL;
  return EA_OK;
}

inline bool empty(const ea_batch *b) {
  return b->n_seqs == 0 || b->n_rows == 0 || b->max_rows == 0;
}

inline int check_rows(const ea_rows &r) {
  if (!r.data || !aligned(r.data, 16)) return EA_EINVAL;
  if (r.row_stride % 8 != 0 || r.head_stride % 8 != 0) return EA_EINVAL;
  return EA_OK;
}

inline ea::HeadRows rows(const ea_rows &r) {
  return {static_cast<uint16_t *>(r.data), r.row_stride, r.head_stride};
}

inline ea::BatchRows batch_rows(const ea_batch *b) {
  return {b->page_table, b->kv_len, b->row_start, b->table_stride,
          b->n_seqs,     b->n_rows, b->max_rows,  b->max_kv};
}

inline int check_cache(const ea_cache *c, int32_t dtype) {
  if (!c || (dtype != EA_BF16 && dtype != EA_F16)) return EA_EINVAL;
  const ea_cache_desc &d = ea::cache_desc(c);
  if (d.elem_bytes != 1 && d.elem_bytes != 2) return EA_ENOTSUP;
  if (d.head_dim % 8 != 0 || d.head_dim > ea::kMaxHeadDim) return EA_ENOTSUP;
  if ((int64_t)d.num_pages * d.page_tokens > INT32_MAX) return EA_ENOTSUP;
  // places inside a page are 32 bits
  if (2LL * d.page_tokens * d.num_kv_heads * d.head_dim * d.elem_bytes > (1 << 30))
    return EA_ENOTSUP;
  return EA_OK;
}

// A cache of latents: a token's row in place of one head's key and value.
inline int check_latents(const ea_cache *c, int32_t latent, int32_t turn, int32_t dtype) {
  if (!c || (dtype != EA_BF16 && dtype != EA_F16)) return EA_EINVAL;
  const ea_cache_desc &d = ea::cache_desc(c);
  if (latent < 1 || turn < 1 || d.num_kv_heads != 1 || (int64_t)latent + turn != 2LL * d.head_dim)
    return EA_EINVAL;
  if (d.elem_bytes != 1 && d.elem_bytes != 2) return EA_ENOTSUP;
  if (latent % 16 != 0 || latent > ea::kMaxLatent || turn % 16 != 0 || turn > ea::kMaxTurn)
    return EA_ENOTSUP;
  if ((int64_t)d.num_pages * d.page_tokens > INT32_MAX) return EA_ENOTSUP;
  // places inside a page are 32 bits
  if (2LL * d.page_tokens * d.head_dim * d.elem_bytes > (1 << 30)) return EA_ENOTSUP;
  return EA_OK;
}

// The layer with its planes.  Scales: of a block and head, or the cache's
// own one for a block.
inline int layer_of(const ea_cache *c, const ea_cache_planes *planes, int32_t layer,
                    ea::KvLayer *out) {
  const ea_cache_desc &d = ea::cache_desc(c);
  if (layer < 0 || layer >= d.num_layers) return EA_EINVAL;
  ea::KvLayer k{};
  k.num_pages = d.num_pages;
  k.page_tokens = d.page_tokens;
  k.heads = d.num_kv_heads;
  k.head_dim = d.head_dim;
  k.piece = 2LL * d.page_tokens * d.num_kv_heads * d.head_dim * d.elem_bytes;
  k.base = static_cast<uint8_t *>(d.base) + k.piece * d.num_pages * layer;
  // token / T for tokens below 2^31 by a multiplication: 2^(31+l) / T rounded
  // up, 2^l >= T
  int l = 0;
  while ((1LL << l) < d.page_tokens) ++l;
  k.t_mul = (uint32_t)((1ULL << (31 + l)) / (uint32_t)d.page_tokens + 1);
  k.t_shift = l;
  const int64_t page0 = (int64_t)d.num_pages * layer;
  if (planes && planes->head_scales) {
    if (!aligned(planes->head_scales, 4)) return EA_EINVAL;
    k.scales = planes->head_scales + page0 * 2 * d.num_kv_heads;
    k.scale_page = 2 * d.num_kv_heads;
    k.scale_kv = d.num_kv_heads;
    k.scale_head = 1;
  } else if (d.scale_base) {
    k.scales = static_cast<float *>(d.scale_base) + page0 * 2;
    k.scale_page = 2;
    k.scale_kv = 1;
    k.scale_head = 0;
  }
  if (d.elem_bytes == 1 && !k.scales) return EA_EINVAL;
  if (planes && (planes->bounds || planes->bound_scales)) {
    if (!planes->bounds || !planes->bound_scales) return EA_EINVAL;
    if (!aligned(planes->bounds, 8) || !aligned(planes->bound_scales, 4)) return EA_EINVAL;
    k.bounds = planes->bounds + page0 * 2 * d.num_kv_heads * d.head_dim;
    k.bound_scales = planes->bound_scales + page0 * d.num_kv_heads;
  }
  *out = k;
  return EA_OK;
}

inline int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

// Compute units of a device, asked for once.
inline int compute_units(int dev) {
  static std::atomic<int> known[64];
  if (dev < 0 || dev >= 64) return 256;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
        n < 1)
      n = 256;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

}  // namespace ea::host
