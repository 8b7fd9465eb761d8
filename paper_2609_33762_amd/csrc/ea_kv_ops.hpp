// Shared declarations of the cache operators (append, attention, block
// selection): kernel arguments and launchers.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace ea {

enum Act : int32_t { kBf16 = 0, kF16 = 1 };

// One layer of the paged cache, [P][2][T][H][D], and its planes.
struct KvLayer {
  uint8_t *base;          // first byte of the layer
  float *scales;          // first scale of the layer (fp8), or nullptr
  int8_t *bounds;         // [P][2][H][D] lowest, highest; or nullptr
  float *bound_scales;    // [P][H]
  int64_t piece;          // bytes of one page
  int32_t num_pages, page_tokens, heads, head_dim;
  int32_t scale_page, scale_kv, scale_head;  // strides of `scales` in floats
  // token / page_tokens for 0 <= token < 2^31: the high 32 bits of 2 * token *
  // t_mul, >> t_shift
  uint32_t t_mul;
  int32_t t_shift;
};

// The sequences of one call; every array is device memory.
struct BatchRows {
  const int32_t *page_table;  // [n_seqs][table_stride]
  const int32_t *kv_len;      // [n_seqs]
  const int32_t *row_start;   // [n_seqs + 1], or nullptr: one row each
  int64_t table_stride;
  int32_t n_seqs, n_rows, max_rows, max_kv;
};

// Rows of heads: element (row, head, d) at row * row_stride + head *
// head_stride + d of 16-bit elements.
struct HeadRows {
  uint16_t *data;
  int64_t row_stride, head_stride;
};

struct AppendArgs {
  KvLayer kv;
  BatchRows b;
  HeadRows k, v, q, q_out;  // q.data null: no queries
  const float *rope;        // [rope_len][rope_dim]: cosines, then sines; or nullptr
  int32_t rope_dim, interleaved;
  int32_t q_heads;
  int32_t fp8;
  int32_t pages_most;       // pages one sequence's new tokens can touch
};

struct AttendArgs {
  KvLayer kv;
  BatchRows b;
  HeadRows q, out;
  float *lse;               // [n_rows][q_heads] or nullptr
  const int32_t *selected;  // [n_rows][H][budget] or nullptr
  int32_t budget;
  int32_t window;
  int32_t group;            // query heads per KV head
  float scale_log2;         // softmax scale times log2(e)
  // Sequences with at most this many rows times heads of a group go to the
  // split kernel (0: it is not launched), others to the chunk kernel.
  int32_t split_rows_most;
  // Split kernel: a workgroup takes heads_wg (1 or 2) neighbouring KV heads.
  // A unit (a sequence and as many heads) is split so that the parts of all
  // fit split_wgs workgroups where they can, a part having least_steps steps
  // at least (0: units are not split); split_grid workgroups are enough for
  // that.
  // Their parts, and the counts of a unit's parts done, zero between calls.
  int32_t heads_wg, split_wgs, least_steps, split_grid;
  float *split_parts;
  int32_t *arrivals;
  // Chunk kernel: work along a sequence's tokens in parts of chunk_tokens,
  // `splits` of them at most; launch_attend_join joins a row's parts.
  int32_t splits, chunk_tokens;
  float *part_o;            // [n_rows][q_heads][splits][head_dim]
  float *part_ml;           // [n_rows][q_heads][splits][2]
};

struct SelectArgs {
  KvLayer kv;
  BatchRows b;
  HeadRows q;
  int32_t *selected;        // [n_rows][H][budget]
  uint32_t *keys;           // [n_rows][H][blocks_most] ordered scores
  int32_t budget, first, last;
  int32_t group;
  int32_t blocks_most;      // blocks of max_kv tokens
  int32_t blocks_wave;      // blocks one wave scores
};

// A cache of latents is a KvLayer of one head of half a token's row: a token
// has `latent` elements, then `turn` ones, in place of a key and a value; the
// scales of a block are those of the two parts.
struct LatentAttendArgs {
  KvLayer kv;
  BatchRows b;
  HeadRows q, out;          // [n_rows][q_heads][latent + turn], [n_rows][q_heads][latent]
  float *lse;               // [n_rows][q_heads] or nullptr
  int32_t latent, turn;
  int32_t q_heads;
  float scale_log2;         // softmax scale times log2(e)
  // A workgroup takes 32 * wave_columns (1, 2, 4) rows times heads of a
  // sequence, a unit, at most tiles_most of them a sequence.  Units come in parts
  // so that those of all fit split_wgs workgroups where they can, a part having
  // least_steps steps at least (0: units are not split); split_grid workgroups
  // are enough for that.
  int32_t wave_columns, tiles_most;
  int32_t split_wgs, least_steps, split_grid;
  int32_t *units;           // [n_seqs][tiles_most][2]: a unit's first workgroup, its parts
  float *parts;             // [split_grid][32 * wave_columns][latent, whole 32, + 2]
  int32_t slices;           // workgroups that join a unit's 32 rows; 0: nothing is split
  int32_t two_weights;      // beside bf16 latents: weights are the sum of two bf16
};

struct LatentAppendArgs {
  KvLayer kv;
  BatchRows b;
  HeadRows latents, key;    // [n_rows][1][latent], [n_rows][1][turn]
  HeadRows q, q_out;        // [n_rows][q_heads][turn]; q.data null: no queries
  const float *rope;        // [rope_len][turn]: cosines, then sines; or nullptr
  int32_t latent, turn;
  int32_t interleaved;
  int32_t q_heads;
  int32_t pages_most;       // pages one sequence's new tokens can touch
};

// Kept tokens of sequences on their way to other pages, in `layers` layers from
// kv's on.  Keys and values, or (latent > 0) rows of a latent cache.
struct MoveArgs {
  KvLayer kv;
  int64_t layer_bytes, layer_scales;  // from layer to layer
  const int32_t *src_table, *dst_table;
  int64_t src_stride, dst_stride;
  const int32_t *tokens;        // [n_tokens] old positions
  const int32_t *token_start;   // [n_seqs + 1]
  const int32_t *dst_first;     // [n_seqs] new position of a sequence's first, or nullptr
  const float *rope;            // [rope_len][rope_dim] or nullptr
  int32_t rope_len, rope_dim, interleaved;
  int32_t layers, n_seqs, n_tokens, max_tokens, max_kv;
  int32_t blocks_most;          // blocks of max_tokens
  int32_t layers_wave;          // layers that one wave (workgroup) goes through
  int32_t latent, turn;
};

constexpr int kCopyPlanes = 4;
struct CopyArgs {
  uint8_t *base;
  int64_t piece;
  int32_t num_pages, layers, n;
  int32_t runs_piece;           // runs of a piece, one wave each
  const int32_t *src, *dst;
  uint8_t *plane[kCopyPlanes];  // [layers][num_pages][plane_bytes], or nullptr
  int64_t plane_bytes[kCopyPlanes];
};

// Parts of at most `each` steps that `steps` steps come in.  No sum of the two,
// which could pass 32 bits.
constexpr int32_t parts_of_steps(int32_t steps, int32_t each) {
  return steps > 0 ? (steps - 1) / each + 1 : 0;
}
static_assert(parts_of_steps(0, INT32_MAX) == 0 && parts_of_steps(INT32_MAX, INT32_MAX) == 1 &&
              parts_of_steps(INT32_MAX, 1) == INT32_MAX && parts_of_steps(5, 2) == 3);

// Columns of the split kernel's variant for this many; waves of a variant's
// workgroups, and the workgroups of it that its registers let a compute unit
// hold.
constexpr int32_t split_columns(int32_t most) { return most <= 16 ? 16 : most <= 32 ? 32 : 64; }
constexpr int32_t split_waves(int32_t head_dim, int32_t columns) {
  return head_dim > 128 || columns > 32 ? 4 : 8;
}
constexpr int32_t split_resident(int32_t head_dim, int32_t columns) {
  return head_dim <= 64 && columns <= 16 ? 2 : 1;
}

// Tokens of a step of the latent kernel with this many groups of 32 columns.
constexpr int32_t latent_step(int32_t wave_columns) { return 128 / wave_columns; }

// Counters at the start of an attention workspace: a unit's parts done.  More
// units than kSplitUnits are not split.
constexpr int32_t kSplitUnits = 4096, kArrivals = 8192;

constexpr int32_t kMaxHeadDim = 256;
constexpr int32_t kMaxLatent = 512, kMaxTurn = 64;
constexpr int32_t kMaxSelectBlocks = 65536;

// Most query rows times heads of a group that the split kernel takes (its
// columns per wave); heads wider than 128 leave it fewer registers.
constexpr int32_t split_rows_cap(int32_t head_dim) { return head_dim > 128 ? 16 : 64; }

// Tokens a step of the split kernel covers and rows of a chunk workgroup.
constexpr int32_t kSplitStep = 32;
constexpr int32_t kChunkRows = 128;
constexpr int32_t kChunkTokens = 64;

hipError_t launch_append(const AppendArgs &a, int act, hipStream_t s);
hipError_t launch_bounds(const KvLayer &kv, int act, int fp8, int32_t layers, int64_t layer_bytes,
                         int64_t layer_scales, const int32_t *pages, int32_t n, hipStream_t s);
hipError_t launch_attend_split(const AttendArgs &a, int act, int fp8, hipStream_t s);
hipError_t launch_attend_chunk(const AttendArgs &a, int act, int fp8, hipStream_t s);
hipError_t launch_attend_join(const AttendArgs &a, int act, hipStream_t s);
hipError_t launch_append_latent(const LatentAppendArgs &a, int act, int fp8, hipStream_t s);
hipError_t launch_move_latents(const MoveArgs &a, int act, int fp8, hipStream_t s);
hipError_t launch_move_tokens(const MoveArgs &a, int act, int fp8, hipStream_t s);
int32_t copy_runs(int64_t piece);  // runs of a piece of this many bytes
hipError_t launch_copy_pages(const CopyArgs &a, hipStream_t s);
hipError_t launch_attend_latent(const LatentAttendArgs &a, int act, int fp8, hipStream_t s);
hipError_t launch_select(const SelectArgs &a, int act, hipStream_t s);

}  // namespace ea
