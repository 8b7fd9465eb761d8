// Selection of blocks for sparse attention: a score for every block from
// whole-number bounds of its keys, and the highest ones of each query row
// and KV head.
//
// The largest score a key inside a block's bounds can reach is
//   sum_d max(q_d lo_d, q_d hi_d) = sum_d (max(q_d, 0) hi_d + min(q_d, 0) lo_d),
// a dot product of length 2 D, so it goes to the matrix units.  Bounds and
// query are whole numbers of 8 bits times powers of two: the dot product is
// below 2^24 and the scaled score exact in 32 bits, whatever the order of
// the sum.  That makes the choice, ties and all, a function of its inputs.
#include <hip/hip_runtime.h>

#include "ea_kv_device.hpp"

namespace ea {
namespace {

constexpr int kWaves = 4;

// A float as a whole number of the same order, and the key of a block that
// is always taken.  (-0 is +0.)
__device__ inline uint32_t order_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kAlways = 0xffffffffu;

// One wave: blocks_wave blocks of one query row and KV head.  The bounds of
// 16 blocks are the rows of a product, the heads of the group its columns;
// reading the bounds is what it costs.
template <int ACT>
__global__ __launch_bounds__(kWaves *kLanes) void block_scores(SelectArgs a) {
  const KvLayer &kv = a.kv;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int H = kv.heads, D = kv.head_dim, G = a.group;
  const int waves_row = (a.blocks_most + a.blocks_wave - 1) / a.blocks_wave;
  uint32_t u = blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  const int h = u % H;
  u /= H;
  const int wv = u % waves_row;
  u /= waves_row;
  const int qi = u % a.b.max_rows, s = u / a.b.max_rows;
  if (s >= a.b.n_seqs) return;
  const Seq sq = sequence(a.b, s);
  if (qi >= sq.rows) return;
  const int pos = sq.len - sq.rows + qi, row = sq.row0 + qi;
  if (pos < 0) return;
  const int held = over_page(kv, pos) + 1;  // blocks the row may attend to
  const int b0 = wv * a.blocks_wave, b1 = min(held, b0 + a.blocks_wave);
  if (b0 >= b1) return;
  const int32_t *table = a.b.page_table + (int64_t)s * a.b.table_stride;
  uint32_t *keys = a.keys + ((int64_t)row * H + h) * a.blocks_most;

  constexpr int KS = kMaxHeadDim / 64;  // products a half, at most
  const int ks = (D + 63) / 64;
  for (int g0 = 0; g0 < G; g0 += 16) {  // 16 heads of the group at a time
    const int j = g0 + c;
    // this column's query as whole numbers: elements k * 64 + g * 16 ..+15
    float q[KS][16];
    float amax = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int d = k * 64 + g * 16 + half * 8;
        u32x4 v = {0, 0, 0, 0};
        if (j < G && d < D)
          v = *reinterpret_cast<const u32x4 *>(a.q.data + (int64_t)row * a.q.row_stride +
                                               (int64_t)(h * G + j) * a.q.head_stride + d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = act_to_float<ACT>((uint16_t)(v[i >> 1] >> (16 * (i & 1))));
          q[k][half * 8 + i] = x;
          if (finite(x)) amax = fmaxf(amax, fabsf(x));
        }
      }
    }
    amax = max_rows16(amax);
    const float sq_q = int8_scale(amax), inv = power_inverse(sq_q);
    u32x4 neg[KS], posv[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t n = 0, p = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = rintf(q[k][w * 4 + i] * inv);
          // a NaN counts as zero, an infinity as the largest
          const int v = x == x ? (int)fminf(fmaxf(x, -127.f), 127.f) : 0;
          n |= (uint32_t)(uint8_t)min(v, 0) << (8 * i);
          p |= (uint32_t)(uint8_t)max(v, 0) << (8 * i);
        }
        neg[k][w] = n;
        posv[k][w] = p;
      }
    for (int b = b0; b < b1; b += 16) {
      const int mine = min(b + c, b1 - 1);
      const int pg = table[mine];
      const bool ok = (uint32_t)pg < (uint32_t)kv.num_pages;
      const int page = ok ? pg : 0;
      const int8_t *p = kv.bounds + ((int64_t)page * 2 * H + h) * D;
      const float sb = kv.bound_scales[(int64_t)page * H + h];
      i32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        if (k >= ks) break;
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // lowest, highest
          const int8_t *ph = p + (int64_t)half * H * D;
          const int d = k * 64 + g * 16;
          u32x2 x = {0, 0}, y = {0, 0};  // past the head the query is zero
          if (d < D) x = *reinterpret_cast<const u32x2 *>(ph + d);
          if (d + 8 < D) y = *reinterpret_cast<const u32x2 *>(ph + d + 8);
          acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(
              i32x4{(int)x[0], (int)x[1], (int)y[0], (int)y[1]},
              __builtin_bit_cast(i32x4, half ? posv[k] : neg[k]), acc, 0, 0, 0);
        }
      }
      // result i: block b + g * 4 + i, head j
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float block_scale = __shfl(sb, g * 4 + i);
        const int block_there = __shfl((int)ok, g * 4 + i);
        float v = j < G ? (float)acc[i] * sq_q * block_scale : kNegInf;
        for (int d = 8; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
        const int blk = b + g * 4 + i;
        if (c == i && blk < b1) {
          uint32_t key = order_key(v);
          if (g0) key = max(key, keys[blk]);
          // always taken: the first blocks and the row's last ones; a page
          // that is not there comes after every score
          if (blk < a.first || blk >= held - a.last) key = kAlways;
          else if (!block_there) key = 0;
          keys[blk] = key;
        }
      }
    }
  }
}

// One workgroup of 1024: the budget highest keys of a row and KV head, ties
// to the lowest block, in the blocks' order.  The threads hold the keys in
// registers (PER each); the smallest key taken is found from its highest
// bits down, two at a time, by counting the keys not below three thresholds.
template <int PER>
__global__ __launch_bounds__(1024) void pick_blocks(SelectArgs a) {
  __shared__ int32_t count[2][16][3];
  __shared__ int32_t base_gt[16], base_eq[16];
  const int H = a.kv.heads, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t u = blockIdx.x;
  const int h = u % H;
  u /= H;
  const int qi = u % a.b.max_rows, s = u / a.b.max_rows;
  const Seq sq = sequence(a.b, s);
  if (qi >= sq.rows) return;
  const int pos = sq.len - sq.rows + qi, row = sq.row0 + qi;
  const int held = pos < 0 ? 0 : over_page(a.kv, pos) + 1;
  int32_t *out = a.selected + ((int64_t)row * H + h) * a.budget;
  if (held <= a.budget) {  // all of them
    for (int i = tid; i < a.budget; i += 1024) out[i] = i < held ? i : -1;
    return;
  }
  const uint32_t *keys = a.keys + ((int64_t)row * H + h) * a.blocks_most;
  uint32_t key[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = i * 1024 + tid;
    key[i] = b < held ? keys[b] : 0;
  }
  uint32_t low = 0;  // at least `budget` keys are >= low
  for (int bit = 30, turn = 0; bit >= 0; bit -= 2, turn ^= 1) {
    int n[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool there = i * 1024 + tid < held;
#pragma unroll
      for (int j = 0; j < 3; ++j)
        n[j] += __popcll(__ballot(there && key[i] >= (low | ((uint32_t)(j + 1) << bit))));
    }
    if (lane == 0)
#pragma unroll
      for (int j = 0; j < 3; ++j) count[turn][wave][j] = n[j];
    __syncthreads();
    int total[3] = {0, 0, 0};
#pragma unroll
    for (int w = 0; w < 16; ++w)
#pragma unroll
      for (int j = 0; j < 3; ++j) total[j] += count[turn][w][j];
    uint32_t step = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (total[j] >= a.budget) step = j + 1;
    low |= step << bit;
  }
  // low is the budget-th highest key: all above it are taken, and the first
  // of those equal to it
  int above = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    above += __popcll(__ballot(i * 1024 + tid < held && key[i] > low));
  __syncthreads();
  if (lane == 0) count[0][wave][0] = above;
  __syncthreads();
  above = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) above += count[0][w][0];
  const int equal_room = a.budget - above;
  int gt_before = 0, eq_before = 0;  // over the rounds so far
  for (int i = 0; i < PER; ++i) {
    if (i * 1024 >= held) break;
    const int b = i * 1024 + tid;
    const uint32_t mine = b < held ? keys[b] : 0;
    const bool gt = b < held && mine > low, eq = b < held && mine == low;
    const uint64_t mg = __ballot(gt), me = __ballot(eq);
    __syncthreads();
    if (lane == 0) {
      base_gt[wave] = __popcll(mg);
      base_eq[wave] = __popcll(me);
    }
    __syncthreads();
    int g0 = gt_before, e0 = eq_before;
    for (int w = 0; w < 16; ++w) {
      const int cg = base_gt[w], ce = base_eq[w];
      if (w < wave) {
        g0 += cg;
        e0 += ce;
      }
      gt_before += cg;
      eq_before += ce;
    }
    const uint64_t below = (1ull << lane) - 1;
    g0 += __popcll(mg & below);
    e0 += __popcll(me & below);
    if (gt || (eq && e0 < equal_room)) out[g0 + min(e0, equal_room)] = b;
  }
}

}  // namespace

hipError_t launch_select(const SelectArgs &a, int act, hipStream_t s) {
  (void)hipGetLastError();
  const int64_t rows = (int64_t)a.b.n_seqs * a.b.max_rows * a.kv.heads;
  const int64_t waves = rows * ((a.blocks_most + a.blocks_wave - 1) / a.blocks_wave);
  const dim3 grid((unsigned)((waves + kWaves - 1) / kWaves)), block(kWaves * kLanes);
  if (act == kBf16) hipLaunchKernelGGL(block_scores<kBf16>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(block_scores<kF16>, grid, block, 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 per_row((unsigned)rows), big(1024);
  if (a.blocks_most <= 4 * 1024) hipLaunchKernelGGL(pick_blocks<4>, per_row, big, 0, s, a);
  else if (a.blocks_most <= 16 * 1024) hipLaunchKernelGGL(pick_blocks<16>, per_row, big, 0, s, a);
  else hipLaunchKernelGGL(pick_blocks<64>, per_row, big, 0, s, a);
  return hipGetLastError();
}

}  // namespace ea
