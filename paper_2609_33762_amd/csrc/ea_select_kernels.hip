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
// 16 blocks are the rows of a product, the heads of the group its columns.
// Reading the bounds is what it costs: the next 16 load while these are
// scored, and their pages were looked up before that (64 rows of 4 heads over
// up to 4,096 blocks in 47 us).  KS: products of 64
// elements a half.
template <int ACT, int KS, bool WIDE>
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

  struct Bounds {
    u32x4 x[KS][2];  // lowest, highest
    float scale;
    bool there;
  };
  auto page_of = [&](int b) { return (uint32_t)table[min(b + c, b1 - 1)]; };
  auto load = [&](uint32_t pg) {
    Bounds r;
    r.there = pg < (uint32_t)kv.num_pages;
    const uint32_t page = r.there ? pg : 0;
    r.scale = kv.bound_scales[(uint64_t)page * H + h];
    const int8_t *p = kv.bounds + ((uint64_t)page * 2 * H + h) * D;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        // past the head the query is zero: any bytes serve
        const int d = k * 64 + g * 16;
        const int8_t *ph = p + (int64_t)half * H * D;
        if constexpr (WIDE) {
          r.x[k][half] = *reinterpret_cast<const u32x4 *>(ph + (d < D ? d : 0));
        } else {
          const u32x2 x = *reinterpret_cast<const u32x2 *>(ph + (d < D ? d : 0));
          const u32x2 y = *reinterpret_cast<const u32x2 *>(ph + (d + 8 < D ? d + 8 : 0));
          r.x[k][half] = u32x4{x[0], x[1], y[0], y[1]};
        }
      }
    return r;
  };

  for (int g0 = 0; g0 < G; g0 += 16) {  // 16 heads of the group at a time
    const int j = g0 + c;
    uint32_t page = page_of(b0 + 16);
    Bounds now = load(page_of(b0));
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
      const Bounds next = load(page);
      page = page_of(b + 32);
      i32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int half = 0; half < 2; ++half)
          acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(
              __builtin_bit_cast(i32x4, now.x[k][half]),
              __builtin_bit_cast(i32x4, half ? posv[k] : neg[k]), acc, 0, 0, 0);
      // result i: block b + g * 4 + i, head j; lane c < 4 writes block
      // b + g * 4 + c
      float best = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = max_columns(j < G ? (float)acc[i] * sq_q : kNegInf);
        if (c == i) best = v;
      }
      const int from = g * 4 + (c & 3), blk = b + from;
      const float scale = __shfl(now.scale, from);
      const int there = __shfl((int)now.there, from);
      if (c < 4 && blk < b1) {
        uint32_t key = order_key(best * scale);
        if (g0) key = max(key, keys[blk]);
        // always taken: the first blocks and the row's last ones; a page that
        // is not there comes after every score
        if (blk < a.first || blk >= held - a.last) key = kAlways;
        else if (!there) key = 0;
        keys[blk] = key;
      }
      now = next;
    }
  }
}

// One workgroup: the budget highest keys of a row and KV head, ties to the
// lowest block, in the blocks' order; PER keys a thread.  The lowest key taken
// is found from its highest bits down: a histogram of the eight highest bits
// in which the keys differ, then of the next eight of those in the bin that
// the bound falls into, until a bin is wanted as a whole.  Its latency is the
// few passes over LDS, 8-10 us whatever the number of rows up to the card's
// workgroups.
template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void pick_blocks(SelectArgs a) {
  constexpr int W = THREADS / kLanes;
  __shared__ int32_t count[W][4];
  __shared__ int32_t bins[256], found[3];
  const int H = a.kv.heads, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
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
    for (int i = tid; i < a.budget; i += THREADS) out[i] = i < held ? i : -1;
    return;
  }
  const uint32_t *keys = a.keys + ((int64_t)row * H + h) * a.blocks_most;
  // A place past the blocks holds 0, as does a block whose page is not there;
  // scores are above that.
  constexpr bool kHeld = PER <= 16;  // in registers; else read again
  uint32_t kept[kHeld ? PER : 1];
  auto fetch = [&](int i) {
    const int b = (wave * PER + i) * kLanes + lane;
    return b < held ? keys[b] : 0u;
  };
  if (kHeld) {
#pragma unroll
    for (int i = 0; i < PER; ++i) kept[kHeld ? i : 0] = fetch(i);
  }
  auto key = [&](int i) { return kHeld ? kept[kHeld ? i : 0] : fetch(i); };
  uint32_t any = 0, all = ~0u;
  int forced = 0, scored = 0;
#pragma unroll kHeld ? PER : 4
  for (int i = 0; i < PER; ++i) {
    const uint32_t k = key(i);
    const bool plain = k != kAlways && k != 0;
    if (plain) {
      any |= k;
      all &= k;
    }
    scored += __popcll(__ballot(plain));
    forced += __popcll(__ballot(k == kAlways));
  }
  for (int d = 32; d; d >>= 1) {
    any |= __shfl_xor(any, d);
    all &= __shfl_xor(all, d);
  }
  if (lane == 0) {
    count[wave][0] = (int32_t)any;
    count[wave][1] = (int32_t)all;
    count[wave][2] = scored;
    count[wave][3] = forced;
  }
  if (tid < 256) bins[tid] = 0;
  __syncthreads();
  scored = forced = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    any |= (uint32_t)count[w][0];
    all &= (uint32_t)count[w][1];
    scored += count[w][2];
    forced += count[w][3];
  }
  // low: keys above it are taken, and of those equal to it what there is room
  // for
  uint32_t low = 0;  // too few scores: all of them, then blocks without a page
  int wanted = a.budget - forced;  // of the scored ones
  if (wanted <= 0) {
    low = kAlways;
  } else if (wanted < scored) {
    const uint32_t differ = any & ~all;
    int bits = differ ? 32 - __builtin_clz(differ) : 0;  // still to be told apart
    uint32_t prefix = bits < 32 ? all >> bits : 0;       // above them
    while (bits > 0) {
      const int width = min(bits, 8), shift = bits - width;
#pragma unroll kHeld ? PER : 4
      for (int i = 0; i < PER; ++i) {
        const uint32_t k = key(i);
        if (k != kAlways && k != 0 && (bits == 32 || k >> bits == prefix))
          atomicAdd(&bins[(k >> shift) & ((1u << width) - 1)], 1);
      }
      __syncthreads();
      // keys in a bin or above it: thread t has bin 255 - t
      const int in = tid < 256 ? bins[255 - tid] : 0;
      const int upto = scan_wave(in);
      if (lane == 63) count[wave][0] = upto;
      __syncthreads();
      if (tid < 256) {
        bins[tid] = 0;
        int from = upto;
        for (int w = 0; w < wave; ++w) from += count[w][0];
        if (from >= wanted && from - in < wanted) {
          found[0] = 255 - tid;
          found[1] = from - in;
          found[2] = in;
        }
      }
      __syncthreads();
      prefix = (prefix << width) | (uint32_t)found[0];
      wanted -= found[1];
      bits = shift;
      if (found[2] == wanted) break;
    }
    // the keys from prefix << bits on, or that key itself with room for
    // `wanted` of its blocks
    low = prefix << bits;
    if (bits > 0 && low > 0) --low;
  }
  // Taken are the keys above low and the first of those equal to it that there
  // is room for.  Wave w holds blocks w * PER * 64 on.
  int gt = 0, eq = 0;
#pragma unroll kHeld ? PER : 4
  for (int i = 0; i < PER; ++i) {
    const uint32_t k = key(i);
    gt += __popcll(__ballot(k > low));
    eq += __popcll(__ballot(k == low && (wave * PER + i) * kLanes + lane < held));
  }
  __syncthreads();  // the last counts have been read
  if (lane == 0) {
    count[wave][0] = gt;
    count[wave][1] = eq;
  }
  __syncthreads();
  int above = 0, gt_at = 0, eq_at = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    above += count[w][0];
    if (w < wave) {
      gt_at += count[w][0];
      eq_at += count[w][1];
    }
  }
  const int room = a.budget - above;
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll kHeld ? PER : 4
  for (int i = 0; i < PER; ++i) {
    const int b = (wave * PER + i) * kLanes + lane;
    const uint32_t k = key(i);
    const uint64_t mg = __ballot(k > low), me = __ballot(k == low && b < held);
    const int g0 = gt_at + __popcll(mg & below), e0 = eq_at + __popcll(me & below);
    if (b < held && (k > low || (k == low && e0 < room))) out[g0 + min(e0, room)] = b;
    gt_at += __popcll(mg);
    eq_at += __popcll(me);
  }
}

template <int ACT, int KS>
void scores_of(const SelectArgs &a, dim3 grid, dim3 block, hipStream_t s) {
  // 16 elements at a time where heads are whole pieces of them
  if (a.kv.head_dim % 16 == 0 && (reinterpret_cast<uintptr_t>(a.kv.bounds) & 15) == 0)
    hipLaunchKernelGGL((block_scores<ACT, KS, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((block_scores<ACT, KS, false>), grid, block, 0, s, a);
}

template <int ACT>
void scores(const SelectArgs &a, dim3 grid, dim3 block, hipStream_t s) {
  if (a.kv.head_dim <= 64) scores_of<ACT, 1>(a, grid, block, s);
  else if (a.kv.head_dim <= 128) scores_of<ACT, 2>(a, grid, block, s);
  else scores_of<ACT, 4>(a, grid, block, s);
}

}  // namespace

hipError_t launch_select(const SelectArgs &a, int act, hipStream_t s) {
  (void)hipGetLastError();
  const int64_t rows = (int64_t)a.b.n_seqs * a.b.max_rows * a.kv.heads;
  const int64_t waves = rows * ((a.blocks_most + a.blocks_wave - 1) / a.blocks_wave);
  const dim3 grid((unsigned)((waves + kWaves - 1) / kWaves)), block(kWaves * kLanes);
  if (act == kBf16) scores<kBf16>(a, grid, block, s);
  else scores<kF16>(a, grid, block, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 per_row((unsigned)rows);
  if (a.blocks_most <= 256 * 4)
    hipLaunchKernelGGL((pick_blocks<256, 4>), per_row, dim3(256), 0, s, a);
  else if (a.blocks_most <= 256 * 16)
    hipLaunchKernelGGL((pick_blocks<256, 16>), per_row, dim3(256), 0, s, a);
  else if (a.blocks_most <= 1024 * 16)
    hipLaunchKernelGGL((pick_blocks<1024, 16>), per_row, dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL((pick_blocks<1024, 64>), per_row, dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace ea
