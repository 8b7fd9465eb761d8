// Entry points of what is done to a cache's pages (include/ea.h): validation
// and the launches.  They allocate nothing.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <climits>
#include <cstdint>

#include "ea.h"
#include "ea_internal.hpp"
#include "ea_kv_host.hpp"
#include "ea_kv_ops.hpp"

using namespace ea::host;

extern "C" {

int ea_copy_pages(ea_cache *c, const ea_cache_planes *planes, const int32_t *d_src,
                  const int32_t *d_dst, int32_t n, hipStream_t stream) {
  if (!c || n < 0) return EA_EINVAL;
  if (planes && (!aligned(planes->head_scales, 4) || !aligned(planes->bound_scales, 4)))
    return EA_EINVAL;
  if (n == 0) return EA_OK;
  if (!d_src || !d_dst || !aligned(d_src, 4) || !aligned(d_dst, 4)) return EA_EINVAL;
  const ea_cache_desc &d = ea::cache_desc(c);
  ea::CopyArgs k{};
  k.base = static_cast<uint8_t *>(d.base);
  k.piece = 2LL * d.page_tokens * d.num_kv_heads * d.head_dim * d.elem_bytes;
  k.num_pages = d.num_pages;
  k.layers = d.num_layers;
  k.n = n;
  k.src = d_src;
  k.dst = d_dst;
  const int64_t heads = d.num_kv_heads;
  k.plane[0] = static_cast<uint8_t *>(d.scale_base);
  k.plane_bytes[0] = 8;
  if (planes) {
    k.plane[1] = reinterpret_cast<uint8_t *>(planes->head_scales);
    k.plane_bytes[1] = 8 * heads;
    k.plane[2] = reinterpret_cast<uint8_t *>(planes->bounds);
    k.plane_bytes[2] = 2 * heads * d.head_dim;
    k.plane[3] = reinterpret_cast<uint8_t *>(planes->bound_scales);
    k.plane_bytes[3] = 4 * heads;
  }
  // runs of a wave, and workgroups, are counted in 32 bits
  if (k.piece > (1LL << 40)) return EA_ENOTSUP;
  k.runs_piece = ea::copy_runs(k.piece);
  if ((int64_t)n * d.num_layers > INT32_MAX / ((int64_t)k.runs_piece + 1)) return EA_ENOTSUP;
  OnDevice on(ea::cache_device(c));
  KV_HIP(on.status());
  KV_HIP(ea::launch_copy_pages(k, stream));
  return EA_OK;
}

int ea_move_tokens(ea_cache *c, const ea_cache_planes *planes, int32_t layer_begin,
                   int32_t layer_count, const ea_move *a, hipStream_t stream) {
  if (!a) return EA_EINVAL;
  const bool latents = a->latent_dim != 0;
  KV_TRY(latents ? check_latents(c, a->latent_dim, a->rope_dim, a->dtype)
                 : check_cache(c, a->dtype));
  const ea_cache_desc &d = ea::cache_desc(c);
  if (layer_begin < 0 || layer_count < 0 || (int64_t)layer_begin + layer_count > d.num_layers)
    return EA_EINVAL;
  if (a->n_seqs < 0 || a->n_tokens < 0 || a->max_tokens < 0 || a->max_kv < 0) return EA_EINVAL;
  if (layer_count == 0 || a->n_seqs == 0 || a->n_tokens == 0 || a->max_tokens == 0) return EA_OK;
  if (!a->src_table || !a->dst_table || !a->tokens || !a->token_start) return EA_EINVAL;
  if (!aligned(a->src_table, 4) || !aligned(a->dst_table, 4) || !aligned(a->tokens, 4) ||
      !aligned(a->token_start, 4) || !aligned(a->dst_first, 4))
    return EA_EINVAL;
  if (a->max_kv < 1 || a->max_kv > (1 << 30) || a->max_tokens > (1 << 30)) return EA_EINVAL;
  const int64_t T = d.page_tokens;
  if (a->src_stride < (a->max_kv + T - 1) / T || a->dst_stride < (a->max_tokens + T - 1) / T ||
      a->src_stride > INT32_MAX || a->dst_stride > INT32_MAX)
    return EA_EINVAL;
  if (a->rope) {
    if (!aligned(a->rope, 16) || a->rope_len < 1) return EA_EINVAL;
    if (!latents &&
        (a->rope_dim < 2 || a->rope_dim % 2 != 0 || a->rope_dim > d.head_dim))
      return EA_EINVAL;
  }
  ea::MoveArgs k{};
  KV_TRY(layer_of(c, latents ? nullptr : planes, layer_begin, &k.kv));
  k.layer_bytes = k.kv.piece * d.num_pages;
  k.layer_scales = (int64_t)d.num_pages * k.kv.scale_page;
  // one scale for all heads of a block would have the heads wait for another
  if (!latents && d.elem_bytes == 1 && k.kv.scale_head == 0 && d.num_kv_heads > 1)
    return EA_ENOTSUP;
  k.src_table = a->src_table;
  k.dst_table = a->dst_table;
  k.src_stride = a->src_stride;
  k.dst_stride = a->dst_stride;
  k.tokens = a->tokens;
  k.token_start = a->token_start;
  k.dst_first = a->dst_first;
  k.rope = a->rope;
  k.rope_len = a->rope_len;
  k.rope_dim = a->rope_dim;
  k.interleaved = a->interleaved;
  k.layers = layer_count;
  k.n_seqs = a->n_seqs;
  k.n_tokens = a->n_tokens;
  k.max_tokens = a->max_tokens;
  k.max_kv = a->max_kv;
  // 16-bit latents go 16 tokens at a time, whatever block they are in
  const int64_t unit = latents && d.elem_bytes == 2 ? 16 : T;
  k.blocks_most = (int32_t)((a->max_tokens + unit - 1) / unit);
  const int64_t blocks = (int64_t)a->n_seqs * k.blocks_most;
  // As many layers as leave 8,192 waves, since lookups and angles serve all of them: two
  // layers of 16 and of 8 long contexts 420 and 205 us, one at a time 440 and 244; of
  // one short context 5.0 us one at a time, both 6.7.
  k.layers_wave = (int32_t)std::min<int64_t>(
      layer_count, std::max<int64_t>(1, blocks * layer_count / 8192));
  k.latent = a->latent_dim;
  k.turn = a->rope_dim;
  // workgroups and waves are counted in 32 bits
  if (blocks > INT32_MAX / layer_count) return EA_ENOTSUP;
  OnDevice on(ea::cache_device(c));
  KV_HIP(on.status());
  const int fp8 = d.elem_bytes == 1;
  KV_HIP(latents ? ea::launch_move_latents(k, a->dtype, fp8, stream)
                 : ea::launch_move_tokens(k, a->dtype, fp8, stream));
  return EA_OK;
}

}  // extern "C"
