// Entry points of the latent cache (include/ea.h): validation, the split of an
// attention call along the tokens, and the launches.  They allocate nothing.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>

#include "ea.h"
#include "ea_internal.hpp"
#include "ea_kv_host.hpp"
#include "ea_kv_ops.hpp"

using namespace ea::host;

namespace {

// How an attention call is split along its tokens, and its workspace: where the
// units' parts are, the parts.
struct Parts {
  int32_t wave_columns, tiles, wgs, least_steps, grid, slices;
  int64_t unit_bytes, bytes;
};

Parts parts_of(const ea_cache *c, const ea_batch *b, const ea_latent_attention *a) {
  Parts p{};
  const int64_t most = (int64_t)b->max_rows * a->q_heads;
  const int cus = compute_units(ea::cache_device(c));
  const bool fp8 = ea::cache_desc(c).elem_bytes == 1;
  // As few waves on other columns of the same tokens as hold the rows times heads:
  // 64 sequences of 8,192-65,536 tokens in fp8, 16 columns: 1, 2, 4 waves 336, 578,
  // 755 us; 64 columns: 2, 4 waves 608, 787; 128 columns: 2, 4 waves 1676, 848.  In
  // 16 bits two waves on the same tokens leave a tile no registers for the queries (24
  // sequences of 2-4 rows of 16 heads: 126 us, with four 101).
  p.wave_columns = !fp8 || most > 64 ? 4 : most > 32 ? 2 : 1;
  const int64_t tile = 32 * p.wave_columns;
  p.tiles = (int32_t)((most + tile - 1) / tile);
  const int64_t units = std::min<int64_t>((int64_t)b->n_seqs * p.tiles,
                                          (int64_t)b->n_rows * a->q_heads / tile + b->n_seqs);
  // A workgroup has a compute unit to itself.  Fewer units than those: one part for
  // each (64 sequences, fp8: 308 us; 1.5 or 2 parts for each: 382, 335), of four steps at
  // least (16: 29 us in place of 18 for 512 tokens, as much for 65,536; 2: 109 in place
  // of 102 for 24 sequences).  Up to twice as many: long ones are split, so that no compute unit
  // gets two of them (300 sequences of 500-16,000 tokens: 387 us, whole 426, four
  // times as many parts 410; bf16: 848, 1000, 817).  More: whole units, one launch.
  p.wgs = units <= cus ? cus : 2 * cus;
  p.least_steps = units <= cus ? 4 : units < p.wgs ? 16 : 0;
  const int64_t step = ea::latent_step(p.wave_columns);
  const int64_t steps = (b->max_kv + step - 1) / step;
  const int64_t whole = p.least_steps ? (steps + p.least_steps - 1) / p.least_steps : 1;
  p.grid = (int32_t)std::min<int64_t>(p.wgs + units, units * whole);
  if (p.grid > units) {
    const int64_t groups = (int64_t)b->n_seqs * p.tiles * p.wave_columns;
    // workgroups that join a unit: most of the time 8 waves each, a piece of 8 elements
    // at a time (512 or 2,048 in all: within 4%; 256: 24 sequences take a third more)
    p.slices = (int32_t)std::min<int64_t>(up(a->latent_dim, 32) / 8,
                                          std::max<int64_t>(1, 1024 / groups));
    p.unit_bytes = up((int64_t)b->n_seqs * p.tiles * 8, 16);
    p.bytes = p.unit_bytes + (int64_t)p.grid * tile * (up(a->latent_dim, 32) + 2) * 4;
  }
  return p;
}

int check_attention(const ea_cache *c, const ea_batch *b, const ea_latent_attention *a) {
  if (!a) return EA_EINVAL;
  KV_TRY(check_latents(c, a->latent_dim, a->rope_dim, a->dtype));
  KV_TRY(check_batch(ea::cache_desc(c), b));
  if (a->q_heads < 1) return EA_EINVAL;
  if (!(a->scale > 0.f) || !std::isfinite(a->scale)) return EA_EINVAL;
  if (empty(b)) return EA_OK;
  // rows times heads, and steps of all units, are counted in 32 bits
  const int64_t most = (int64_t)b->max_rows * a->q_heads;
  if ((int64_t)b->n_rows * a->q_heads > INT32_MAX / 4 || most > INT32_MAX / 4) return EA_ENOTSUP;
  if ((int64_t)b->n_seqs * (most / 32 + 1) > INT32_MAX / (b->max_kv / 32 + 1)) return EA_ENOTSUP;
  return EA_OK;
}

}  // namespace

extern "C" {

int ea_append_latent(ea_cache *c, int32_t layer, const ea_batch *b, const ea_latent_append *a,
                     hipStream_t stream) {
  if (!a) return EA_EINVAL;
  KV_TRY(check_latents(c, a->latent_dim, a->rope_dim, a->dtype));
  const ea_cache_desc &d = ea::cache_desc(c);
  KV_TRY(check_batch(d, b));
  ea::LatentAppendArgs k{};
  KV_TRY(layer_of(c, nullptr, layer, &k.kv));
  if (empty(b)) return EA_OK;
  KV_TRY(check_rows(a->latent));
  KV_TRY(check_rows(a->key));
  if (a->q.data) {
    KV_TRY(check_rows(a->q));
    KV_TRY(check_rows(a->q_out));
    if (a->q_heads < 1) return EA_EINVAL;
    k.q = rows(a->q);
    k.q_out = rows(a->q_out);
    k.q_heads = a->q_heads;
  }
  if (a->rope && (!aligned(a->rope, 16) || a->rope_len < b->max_kv)) return EA_EINVAL;
  k.b = batch_rows(b);
  k.latents = rows(a->latent);
  k.key = rows(a->key);
  k.rope = a->rope;
  k.latent = a->latent_dim;
  k.turn = a->rope_dim;
  k.interleaved = a->interleaved;
  k.pages_most = (int32_t)((b->max_rows + (int64_t)d.page_tokens - 2) / d.page_tokens + 1);
  // workgroups, and waves of queries, are counted in 32 bits
  const int64_t blocks = (int64_t)b->n_seqs * k.pages_most;
  const int64_t queries = (int64_t)b->n_rows * ((int64_t)k.q_heads * k.turn / 1920 + 1);
  if (blocks > INT32_MAX / 2 || queries > INT32_MAX / 2) return EA_ENOTSUP;
  OnDevice on(ea::cache_device(c));
  KV_HIP(on.status());
  KV_HIP(ea::launch_append_latent(k, a->dtype, d.elem_bytes == 1, stream));
  return EA_OK;
}

int64_t ea_attend_latent_workspace(const ea_cache *c, const ea_batch *b,
                                   const ea_latent_attention *a) {
  KV_TRY(check_attention(c, b, a));
  if (empty(b)) return 0;
  return parts_of(c, b, a).bytes;
}

int ea_attend_latent(ea_cache *c, int32_t layer, const ea_batch *b, const ea_latent_attention *a,
                     void *workspace, int64_t workspace_bytes, hipStream_t stream) {
  KV_TRY(check_attention(c, b, a));
  ea::LatentAttendArgs k{};
  KV_TRY(layer_of(c, nullptr, layer, &k.kv));
  if (empty(b)) return EA_OK;
  KV_TRY(check_rows(a->q));
  KV_TRY(check_rows(a->out));
  if (a->lse && !aligned(a->lse, 4)) return EA_EINVAL;
  const Parts p = parts_of(c, b, a);
  if (workspace_bytes < p.bytes || (p.bytes > 0 && (!workspace || !aligned(workspace, 16))))
    return EA_EINVAL;
  k.b = batch_rows(b);
  k.q = rows(a->q);
  k.out = rows(a->out);
  k.lse = a->lse;
  k.latent = a->latent_dim;
  k.turn = a->rope_dim;
  k.q_heads = a->q_heads;
  k.scale_log2 = a->scale * 1.4426950408889634f;
  k.wave_columns = p.wave_columns;
  k.tiles_most = p.tiles;
  k.split_wgs = p.wgs;
  k.least_steps = p.least_steps;
  k.split_grid = p.grid;
  k.units = static_cast<int32_t *>(workspace);
  k.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + p.unit_bytes);
  k.slices = p.slices;
  // Half of the waves have no columns then, and bf16 latents get weights of 16 bits for
  // 0 to 10% of the time (64 sequences of 8,192-65,536 tokens, 16 heads: 689 us with 8
  // bits, 736 with 16; 64 heads: 729, 801; 300 of 500-16,000: 826, 847; one of
  // 65,536: 47.6, 47.8).
  k.two_weights = (int64_t)b->max_rows * a->q_heads <= 64;
  OnDevice on(ea::cache_device(c));
  KV_HIP(on.status());
  KV_HIP(ea::launch_attend_latent(k, a->dtype, ea::cache_desc(c).elem_bytes == 1, stream));
  return EA_OK;
}

}  // extern "C"
