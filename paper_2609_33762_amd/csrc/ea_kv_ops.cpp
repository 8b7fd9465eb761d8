// Entry points of the cache operators (include/ea.h): validation, the split
// of the work along the tokens, and the launches.  They allocate nothing.
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

// How an attention call is split along its tokens, and its workspace: the
// counters, always first, the split kernel's parts, the chunk kernel's parts.
constexpr int64_t kCounters = ea::kArrivals * 4;
struct Parts {
  bool split, chunk;  // kernels to launch
  int32_t heads_wg, split_wgs, least_steps, split_grid;
  int32_t splits, chunk_tokens;
  int64_t split_bytes, chunk_bytes, bytes;  // the last with the counters
};

Parts parts_of(const ea_cache *c, const ea_batch *b, const ea_attention *a) {
  const ea_cache_desc &d = ea::cache_desc(c);
  Parts p{};
  const int64_t H = d.num_kv_heads, G = a->q_heads / H, T = d.page_tokens;
  const int64_t cap = ea::split_rows_cap(d.head_dim);
  int64_t span = b->max_kv;
  if (a->selected) span = std::min<int64_t>(up(span, T), (int64_t)a->budget * T);
  else if (a->window > 0)
    span = std::min<int64_t>(span, (int64_t)a->window + b->max_rows + ea::kChunkTokens);
  p.chunk = !a->selected && b->max_rows * G > cap;
  // where all sequences may have the chunk's rows the split kernel is not
  // launched, and the chunk kernel takes sequences of fewer rows too
  p.split = !p.chunk || (int64_t)b->n_seqs * b->max_rows != b->n_rows;
  p.splits = 1;
  p.chunk_tokens = (int32_t)up(std::max<int64_t>(span, 1) + ea::kChunkTokens, ea::kChunkTokens);
  if (p.split) {
    const int64_t most = (a->selected ? 1 : b->max_rows) * G;
    const int64_t cols = ea::split_columns((int32_t)std::min(most, cap));
    // Two neighbouring heads to a workgroup where a head of a token is less
    // than a cache line, whose other part another compute unit would fetch
    // again; and where there are units enough for the chip, as a token's heads
    // are neighbours in memory too: 16 contexts of 32,768 fp8 tokens and 4
    // heads 103.9 -> 100.4 us, up to 4 drafted rows of 16 contexts with 8 heads
    // 87.5 -> 82.4; one context of 65,536 tokens, whose parts then hold twice
    // the rows, 34.1 -> 39.4; four heads to a workgroup 108, 97 and 46.
    // Selections are a head's own.
    const int32_t waves = ea::split_waves(d.head_dim, (int32_t)cols);
    p.heads_wg = !a->selected && H % 2 == 0 &&
                         (d.head_dim * d.elem_bytes < 128 || b->n_seqs * H >= 64)
                     ? 2
                     : 1;
    const int64_t step = ea::kSplitStep * (waves / p.heads_wg);
    const int64_t steps = (span + ea::kChunkTokens + step - 1) / step;
    const int64_t units = (int64_t)b->n_seqs * (a->selected ? b->max_rows : 1) * (H / p.heads_wg);
    // as many workgroups as the chip holds at once
    p.split_wgs = std::min(compute_units(ea::cache_device(c)) *
                               ea::split_resident(d.head_dim, (int32_t)cols),
                           ea::kArrivals - ea::kSplitUnits);
    p.least_steps = units <= ea::kSplitUnits ? 2 : 0;
    // most parts of a unit
    const int64_t whole = p.least_steps ? (steps + p.least_steps - 1) / p.least_steps : 1;
    p.split_grid = (int32_t)std::min<int64_t>(p.split_wgs + units, units * whole);
    if (p.split_grid > units)
      p.split_bytes = up(p.split_grid * p.heads_wg * cols * (d.head_dim + 2) * 4, 16);
  }
  if (p.chunk) {
    // As many workgroups as the chip holds; twice as many where sequences
    // differ, and then an odd number of parts: workgroups go to the eight XCDs
    // in turn, heads and parts first, and shorter sequences have no last parts,
    // so that even numbers leave XCDs without work.  Six ragged fp8 chunks of
    // one head took 501 us in two parts, 391 in three, 508 in four; twelve of 4
    // heads 395 in one part, 508 in two, 383 in three.
    const int64_t most = b->n_seqs * ((b->max_rows * G + ea::kChunkRows - 1) / ea::kChunkRows);
    const int64_t tiles = std::min(most, (int64_t)b->n_rows * G / ea::kChunkRows + b->n_seqs);
    const int64_t target = 2LL * compute_units(ea::cache_device(c)) * (b->n_seqs > 1 ? 2 : 1);
    int64_t want = std::max<int64_t>(1, (target + H * tiles - 1) / (H * tiles));
    if (b->n_seqs > 1) want |= 1;
    p.chunk_tokens = (int32_t)std::max<int64_t>(up((span + want - 1) / want, ea::kChunkTokens),
                                                512);
    // a span's start is rounded down, which can add a part of the rest
    p.splits = (int32_t)((span + (a->window > 0 ? ea::kChunkTokens : 0) + p.chunk_tokens - 1) /
                         p.chunk_tokens);
    if (p.splits > 1)
      p.chunk_bytes =
          up((int64_t)b->n_rows * a->q_heads * p.splits * (d.head_dim + 2) * 4, 16);
  }
  // whichever kernels run, so that calls of other shapes find the counters zero
  if (p.split_bytes + p.chunk_bytes > 0) p.bytes = kCounters + p.split_bytes + p.chunk_bytes;
  return p;
}

int check_attention(const ea_cache *c, const ea_batch *b, const ea_attention *a) {
  if (!a) return EA_EINVAL;
  KV_TRY(check_cache(c, a->dtype));
  const ea_cache_desc &d = ea::cache_desc(c);
  KV_TRY(check_batch(d, b));
  if (a->q_heads < 1 || a->q_heads % d.num_kv_heads != 0) return EA_EINVAL;
  if (!(a->scale > 0.f) || !std::isfinite(a->scale)) return EA_EINVAL;
  if (a->window < 0 || a->window > (1 << 30)) return EA_EINVAL;
  if (a->selected) {
    if (a->window != 0 || a->budget < 1 || !aligned(a->selected, 4)) return EA_EINVAL;
    if (a->budget > ea::kMaxSelectBlocks) return EA_ENOTSUP;
    if (a->q_heads / d.num_kv_heads > ea::split_rows_cap(d.head_dim)) return EA_ENOTSUP;
    if ((int64_t)a->budget * d.page_tokens > (1 << 30)) return EA_ENOTSUP;
  }
  if (empty(b)) return EA_OK;
  // work items are counted in 32 bits
  const Parts p = parts_of(c, b, a);
  const int64_t H = d.num_kv_heads, G = a->q_heads / H;
  const int64_t tiles = (b->max_rows * G + ea::kChunkRows - 1) / ea::kChunkRows;
  const int64_t units = (int64_t)b->n_seqs * H;
  const int64_t tokens = a->selected ? (int64_t)a->budget * d.page_tokens : b->max_kv;
  if (units > INT32_MAX || (int64_t)b->n_rows * a->q_heads > INT32_MAX) return EA_ENOTSUP;
  if (p.chunk && units * p.splits > INT32_MAX / tiles) return EA_ENOTSUP;
  if (p.split && units * (a->selected ? b->max_rows : 1) > INT32_MAX / (tokens / 128 + 1))
    return EA_ENOTSUP;
  return EA_OK;
}

int check_selection(const ea_cache *c, const ea_batch *b, const ea_selection *a) {
  if (!a) return EA_EINVAL;
  KV_TRY(check_cache(c, a->dtype));
  const ea_cache_desc &d = ea::cache_desc(c);
  KV_TRY(check_batch(d, b));
  if (a->q_heads < 1 || a->q_heads % d.num_kv_heads != 0) return EA_EINVAL;
  if (a->first < 0 || a->last < 0 || a->budget < 1 ||
      (int64_t)a->first + a->last > a->budget)
    return EA_EINVAL;
  if (empty(b)) return EA_OK;
  const int64_t blocks = ((int64_t)b->max_kv + d.page_tokens - 1) / d.page_tokens;
  if (blocks > ea::kMaxSelectBlocks || a->budget > ea::kMaxSelectBlocks) return EA_ENOTSUP;
  if ((int64_t)b->n_seqs * b->max_rows > INT32_MAX / d.num_kv_heads) return EA_ENOTSUP;
  if ((int64_t)b->n_seqs * b->max_rows * d.num_kv_heads > INT32_MAX / (blocks / 16 + 1))
    return EA_ENOTSUP;
  return EA_OK;
}

}  // namespace

extern "C" {

int ea_append_kv(ea_cache *c, const ea_cache_planes *planes, int32_t layer, const ea_batch *b,
                 const ea_append *a, hipStream_t stream) {
  if (!a) return EA_EINVAL;
  KV_TRY(check_cache(c, a->dtype));
  const ea_cache_desc &d = ea::cache_desc(c);
  KV_TRY(check_batch(d, b));
  ea::AppendArgs k{};
  KV_TRY(layer_of(c, planes, layer, &k.kv));
  // one scale for all heads of a block would have the heads wait for another
  if (d.elem_bytes == 1 && k.kv.scale_head == 0 && d.num_kv_heads > 1) return EA_ENOTSUP;
  if (empty(b)) return EA_OK;
  KV_TRY(check_rows(a->k));
  KV_TRY(check_rows(a->v));
  if (a->q.data) {
    KV_TRY(check_rows(a->q));
    KV_TRY(check_rows(a->q_out));
    if (a->q_heads < 1) return EA_EINVAL;
  }
  if (a->rope) {
    if (!aligned(a->rope, 16) || a->rope_dim < 2 || a->rope_dim % 2 != 0 ||
        a->rope_dim > d.head_dim || a->rope_len < b->max_kv)
      return EA_EINVAL;
  }
  k.b = batch_rows(b);
  k.k = rows(a->k);
  k.v = rows(a->v);
  if (a->q.data) {
    k.q = rows(a->q);
    k.q_out = rows(a->q_out);
  }
  k.rope = a->rope;
  k.rope_dim = a->rope_dim;
  k.interleaved = a->interleaved;
  k.q_heads = a->q_heads;
  k.fp8 = d.elem_bytes == 1;
  k.pages_most = (int32_t)((b->max_rows + (int64_t)d.page_tokens - 2) / d.page_tokens + 1);
  const int64_t units = (int64_t)b->n_seqs * k.pages_most;
  const int64_t queries = a->q.data ? (int64_t)b->n_rows * (a->q_heads / 16 + 1) : 0;
  if (units > INT32_MAX / (2LL * d.num_kv_heads) ||
      units * 2 * d.num_kv_heads + queries > INT32_MAX)
    return EA_ENOTSUP;
  OnDevice on(ea::cache_device(c));
  KV_HIP(on.status());
  KV_HIP(ea::launch_append(k, a->dtype, stream));
  return EA_OK;
}

int ea_bound_blocks(ea_cache *c, const ea_cache_planes *planes, int32_t layer_begin,
                    int32_t layer_count, const int32_t *d_pages, int32_t n, int32_t dtype,
                    hipStream_t stream) {
  KV_TRY(check_cache(c, dtype));
  const ea_cache_desc &d = ea::cache_desc(c);
  if (n < 0 || layer_begin < 0 || layer_count < 0 ||
      (int64_t)layer_begin + layer_count > d.num_layers)
    return EA_EINVAL;
  if (!planes || !planes->bounds) return EA_EINVAL;
  if (n == 0 || layer_count == 0) return EA_OK;
  if (!d_pages || !aligned(d_pages, 4)) return EA_EINVAL;
  ea::KvLayer k;
  KV_TRY(layer_of(c, planes, layer_begin, &k));
  if ((int64_t)n * layer_count > INT32_MAX / d.num_kv_heads) return EA_ENOTSUP;
  OnDevice on(ea::cache_device(c));
  KV_HIP(on.status());
  KV_HIP(ea::launch_bounds(k, dtype, d.elem_bytes == 1, layer_count, k.piece * d.num_pages,
                           (int64_t)d.num_pages * k.scale_page, d_pages, n, stream));
  return EA_OK;
}

int64_t ea_attend_workspace(const ea_cache *c, const ea_batch *b, const ea_attention *a) {
  KV_TRY(check_attention(c, b, a));
  if (empty(b)) return 0;
  return parts_of(c, b, a).bytes;
}

int ea_attend(ea_cache *c, const ea_cache_planes *planes, int32_t layer, const ea_batch *b,
              const ea_attention *a, void *workspace, int64_t workspace_bytes,
              hipStream_t stream) {
  KV_TRY(check_attention(c, b, a));
  const ea_cache_desc &d = ea::cache_desc(c);
  ea::AttendArgs k{};
  KV_TRY(layer_of(c, planes, layer, &k.kv));
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
  k.selected = a->selected;
  k.budget = a->budget;
  k.window = a->window;
  k.group = a->q_heads / d.num_kv_heads;
  k.scale_log2 = a->scale * 1.4426950408889634f;
  k.split_rows_most = p.split ? ea::split_rows_cap(d.head_dim) : 0;
  k.split_wgs = p.split_wgs;
  k.least_steps = p.least_steps;
  k.split_grid = p.split_grid;
  k.heads_wg = p.heads_wg;
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  k.arrivals = reinterpret_cast<int32_t *>(ws);
  k.split_parts = reinterpret_cast<float *>(ws + kCounters);
  k.splits = p.splits;
  k.chunk_tokens = p.chunk_tokens;
  k.part_o = reinterpret_cast<float *>(ws + kCounters + p.split_bytes);
  k.part_ml = k.part_o + (int64_t)b->n_rows * a->q_heads * p.splits * d.head_dim;
  const int fp8 = d.elem_bytes == 1;
  OnDevice on(ea::cache_device(c));
  KV_HIP(on.status());
  if (p.split) KV_HIP(ea::launch_attend_split(k, a->dtype, fp8, stream));
  if (p.chunk) KV_HIP(ea::launch_attend_chunk(k, a->dtype, fp8, stream));
  if (p.splits > 1) KV_HIP(ea::launch_attend_join(k, a->dtype, stream));
  return EA_OK;
}

int64_t ea_select_workspace(const ea_cache *c, const ea_batch *b, const ea_selection *a) {
  KV_TRY(check_selection(c, b, a));
  if (empty(b)) return 0;
  const ea_cache_desc &d = ea::cache_desc(c);
  const int64_t blocks = ((int64_t)b->max_kv + d.page_tokens - 1) / d.page_tokens;
  return up((int64_t)b->n_rows * d.num_kv_heads * blocks * 4, 16);
}

int ea_select_blocks(ea_cache *c, const ea_cache_planes *planes, int32_t layer,
                     const ea_batch *b, const ea_selection *a, void *workspace,
                     int64_t workspace_bytes, hipStream_t stream) {
  KV_TRY(check_selection(c, b, a));
  const ea_cache_desc &d = ea::cache_desc(c);
  ea::SelectArgs k{};
  KV_TRY(layer_of(c, planes, layer, &k.kv));
  if (!k.kv.bounds) return EA_EINVAL;
  if (empty(b)) return EA_OK;
  KV_TRY(check_rows(a->q));
  if (!a->selected || !aligned(a->selected, 4)) return EA_EINVAL;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < ea_select_workspace(c, b, a))
    return EA_EINVAL;
  k.b = batch_rows(b);
  k.q = rows(a->q);
  k.selected = a->selected;
  k.keys = static_cast<uint32_t *>(workspace);
  k.budget = a->budget;
  k.first = a->first;
  k.last = a->last;
  k.group = a->q_heads / d.num_kv_heads;
  k.blocks_most = (int32_t)(((int64_t)b->max_kv + d.page_tokens - 1) / d.page_tokens);
  // about 16,384 waves (contexts differ in length), each with 16 blocks at
  // least: 64 rows, 4 heads and up to 4,096 blocks 47 us, with 4,096 waves 55
  const int64_t rows_heads = (int64_t)b->n_seqs * b->max_rows * d.num_kv_heads;
  k.blocks_wave = (int32_t)std::max<int64_t>(
      16, up((rows_heads * k.blocks_most + 16383) / 16384, 16));
  OnDevice on(ea::cache_device(c));
  KV_HIP(on.status());
  KV_HIP(ea::launch_select(k, a->dtype, stream));
  return EA_OK;
}

}  // extern "C"
