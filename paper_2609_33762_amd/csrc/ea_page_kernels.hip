// Pages from place to place in a cache: whole pages copied in every layer, and
// tokens of edited contexts moved together into other pages, their keys turned
// from the old position to the new one.
//
// What bounds both is memory: each byte is read once and written once.
#include <hip/hip_runtime.h>

#include "ea_kv_blocks.hpp"
#include "ea_kv_device.hpp"

namespace ea {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kLanes;
constexpr int kLoads = 4;                        // 16-byte loads of a lane
constexpr int64_t kRun = kLoads * kLanes * 16;   // bytes of a piece that a wave copies

// `bytes` from src to dst by a wave, words of `W` bytes.
template <typename W>
__device__ inline void copy_words(uint8_t *dst, const uint8_t *src, int64_t bytes, int lane) {
  for (int64_t i = lane * (int64_t)sizeof(W); i < bytes; i += kLanes * sizeof(W))
    *reinterpret_cast<W *>(dst + i) = *reinterpret_cast<const W *>(src + i);
}

__global__ __launch_bounds__(kThreads) void copy_pages(CopyArgs a, int64_t runs, int64_t units) {
  const int lane = threadIdx.x & 63;
  int64_t u = (int64_t)blockIdx.x * kWaves + uniform((int)threadIdx.x >> 6);
  if (u >= units) return;
  const bool planes = u >= runs;
  if (planes) u -= runs;
  const int per = planes ? 1 : a.runs_piece;
  const int run = u % per;
  u /= per;
  const int layer = u % a.layers, i = u / a.layers;
  const int src = a.src[i], dst = a.dst[i];
  if ((uint32_t)src >= (uint32_t)a.num_pages || (uint32_t)dst >= (uint32_t)a.num_pages) return;
  const int64_t from = (int64_t)layer * a.num_pages + src, to = (int64_t)layer * a.num_pages + dst;
  if (!planes) {
    const int64_t at = run * kRun + lane * 16;
    const u32x4 *p = reinterpret_cast<const u32x4 *>(a.base + from * a.piece + at);
    u32x4 *q = reinterpret_cast<u32x4 *>(a.base + to * a.piece + at);
    u32x4 v[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (at + k * (kRun / kLoads) < a.piece) v[k] = p[k * kLanes];
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (at + k * (kRun / kLoads) < a.piece) q[k * kLanes] = v[k];
    return;
  }
#pragma unroll
  for (int k = 0; k < kCopyPlanes; ++k) {
    uint8_t *b = a.plane[k];
    if (!b) continue;
    const int64_t n = a.plane_bytes[k];
    uint8_t *q = b + to * n;
    const uint8_t *p = b + from * n;
    if (((n | (uintptr_t)b) & 7) == 0) copy_words<u32x2>(q, p, n, lane);
    else if (((n | (uintptr_t)b) & 3) == 0) copy_words<uint32_t>(q, p, n, lane);
    else copy_words<uint8_t>(q, p, n, lane);
  }
}

// A lane's elements of a stored head in 32 bits, turned by |position| `at`
// where rope is not null.
template <int ACT, bool FP8>
__device__ inline void turned(const uint8_t *head, const Place &p, const float *rope, int at,
                              float sign, int dim, bool interleaved, float scale, float x[16]) {
#pragma clang fp contract(off)
  constexpr int EB = FP8 ? 1 : 2;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    if (p.in[n]) {
      stored8<ACT, FP8>(head + p.d[n] * EB, scale, x + n * 8);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[n * 8 + i] = 0.f;
    }
  }
  if (!rope) return;
  const int half = dim >> 1;
  const float *cs = rope + (int64_t)at * dim, *sn = cs + half;
  if (p.paired) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float co = cs[p.d[0] + i], si = sn[p.d[0] + i] * sign, a = x[i], b = x[8 + i];
      const float ac = a * co, bs = b * si, bc = b * co, as = a * si;
      x[i] = ac - bs;
      x[8 + i] = bc + as;
    }
    return;
  }
  auto one = [&](int d) {  // element d as it is stored
    if constexpr (FP8) {
      const f32x2 v = __builtin_amdgcn_cvt_pk_f32_fp8(head[d], false);
      return v[0] * scale;
    } else {
      return act_to_float<ACT>(reinterpret_cast<const uint16_t *>(head)[d]);
    }
  };
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    if (!p.in[n] || p.d[n] >= dim) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = p.d[n] + i;
      if (d >= dim) break;
      const bool upper = interleaved ? d & 1 : d >= half;
      const int f = interleaved ? d >> 1 : upper ? d - half : d;
      const float y = one(interleaved ? d ^ 1 : upper ? d - half : d + half);
      const float xc = x[n * 8 + i] * cs[f], ys = y * (sn[f] * sign);
      x[n * 8 + i] = upper ? xc + ys : xc - ys;
    }
  }
}

// One wave: one block of one layer, for one KV head, keys or values.
template <int ACT, bool FP8, int LP>
__global__ __launch_bounds__(kThreads) void move_tokens(MoveArgs a, int64_t units) {
  constexpr int EB = FP8 ? 1 : 2, TW = kLanes / LP;  // tokens of a pass
  constexpr int KEEP = 2;  // passes whose tokens stay in registers
  const int lane = threadIdx.x & 63;
  int64_t u = (int64_t)blockIdx.x * kWaves + uniform((int)threadIdx.x >> 6);
  if (u >= units) return;
  KvLayer kv = a.kv;
  const int H = kv.heads, D = kv.head_dim;
  const int h = u % H;
  u /= H;
  const bool value = u & 1;
  u >>= 1;
  const int j = u % a.blocks_most;
  u /= a.blocks_most;
  const int s = u % a.n_seqs;
  const int64_t layer = u / a.n_seqs;
  const MovedBlock m = moved_block(a, s, j);
  if (m.n <= 0) return;
  kv.base += layer * a.layer_bytes;
  if (FP8) kv.scales += layer * a.layer_scales;
  if (kv.bounds) {
    kv.bounds += layer * kv.num_pages * 2 * H * D;
    kv.bound_scales += layer * kv.num_pages * H;
  }
  const int64_t token_bytes = (int64_t)H * D * EB;
  const int t0 = lane / LP;
  const float *rope = value ? nullptr : a.rope;
  const Place at = place_of(lane % LP, D, rope != nullptr, a.rope_dim, a.interleaved);
  const int64_t head_at = (value ? kv.piece >> 1 : 0) + (int64_t)h * D * EB;
  uint8_t *dst = kv.base + m.page * kv.piece + head_at;
  auto fetch = [&](int i, float x[16]) {
    const MovedToken t = moved_token(a, m, i);
    if (t.page < 0) {
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] = 0.f;
      return;
    }
    float scale = 1.f;
    if (FP8)
      scale = kv.scales[(int64_t)t.page * kv.scale_page + (value ? kv.scale_kv : 0) +
                        h * kv.scale_head];
    turned<ACT, FP8>(kv.base + t.page * kv.piece + head_at + t.slot * token_bytes, at,
                     t.by ? rope : nullptr, abs(t.by), t.by < 0 ? -1.f : 1.f, a.rope_dim,
                     a.interleaved, scale, x);
  };
  float x[KEEP][16];
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (t0 + k * TW < m.n) fetch(t0 + k * TW, x[k]);
  float scale = 1.f, inv = 1.f;
  if constexpr (FP8) {
    float amax = 0.f;
    auto largest = [&](const float y[16]) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (finite(y[i])) amax = fmaxf(amax, fabsf(y[i]));
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
      if (t0 + k * TW < m.n) largest(x[k]);
    for (int t = t0 + KEEP * TW; t < m.n; t += TW) {
      float y[16];
      fetch(t, y);
      largest(y);
    }
    scale = fp8_scale(max_wave(amax));
    inv = power_inverse(scale);
    if (lane == 0)
      kv.scales[(int64_t)m.page * kv.scale_page + (value ? kv.scale_kv : 0) + h * kv.scale_head] =
          scale;
  }
  const bool bounds = !value && kv.bounds;
  float lo[16], hi[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    lo[i] = __builtin_inff();
    hi[i] = kNegInf;
  }
  auto store = [&](int t, const float y[16]) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      if (!at.in[n]) continue;
      uint8_t *q = dst + t * token_bytes + at.d[n] * EB;
      float z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = FP8 ? y[n * 8 + i] * inv : y[n * 8 + i];
      if constexpr (FP8) {
        const u32x2 w = {fp8_word(z[0], z[1], z[2], z[3]), fp8_word(z[4], z[5], z[6], z[7])};
        *reinterpret_cast<u32x2 *>(q) = w;
        fp8_values(w[0], z);
        fp8_values(w[1], z + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= scale;
      } else {
        const u32x4 w = {pack_act<ACT>(z[0], z[1]), pack_act<ACT>(z[2], z[3]),
                         pack_act<ACT>(z[4], z[5]), pack_act<ACT>(z[6], z[7])};
        *reinterpret_cast<u32x4 *>(q) = w;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          z[i] = act_to_float<ACT>((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
      }
      if (bounds) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          lo[n * 8 + i] = fminf(lo[n * 8 + i], z[i]);
          hi[n * 8 + i] = fmaxf(hi[n * 8 + i], z[i]);
        }
      }
    }
  };
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (t0 + k * TW < m.n) store(t0 + k * TW, x[k]);
  for (int t = t0 + KEEP * TW; t < m.n; t += TW) {
    float y[16];
    fetch(t, y);
    store(t, y);
  }
  if (bounds) write_bounds<LP>(kv, m.page, h, lane, at, lo, hi);
}

template <int ACT, bool FP8>
hipError_t move(const MoveArgs &a, hipStream_t s) {
  const int64_t units = (int64_t)a.layers * a.n_seqs * a.blocks_most * 2 * a.kv.heads;
  const dim3 grid((unsigned)((units + kWaves - 1) / kWaves)), block(kThreads);
  switch (lanes_of(a.kv.head_dim)) {
    case 4: hipLaunchKernelGGL((move_tokens<ACT, FP8, 4>), grid, block, 0, s, a, units); break;
    case 8: hipLaunchKernelGGL((move_tokens<ACT, FP8, 8>), grid, block, 0, s, a, units); break;
    default: hipLaunchKernelGGL((move_tokens<ACT, FP8, 16>), grid, block, 0, s, a, units);
  }
  return hipGetLastError();
}

}  // namespace

int32_t copy_runs(int64_t piece) { return (int32_t)((piece + kRun - 1) / kRun); }

hipError_t launch_copy_pages(const CopyArgs &a, hipStream_t s) {
  (void)hipGetLastError();
  const int64_t runs = (int64_t)a.n * a.layers * a.runs_piece;
  bool planes = false;
  for (int k = 0; k < kCopyPlanes; ++k) planes = planes || a.plane[k];
  const int64_t units = runs + (planes ? (int64_t)a.n * a.layers : 0);
  hipLaunchKernelGGL(copy_pages, dim3((unsigned)((units + kWaves - 1) / kWaves)), dim3(kThreads),
                     0, s, a, runs, units);
  return hipGetLastError();
}

hipError_t launch_move_tokens(const MoveArgs &a, int act, int fp8, hipStream_t s) {
  (void)hipGetLastError();
  if (fp8) return move<kBf16, true>(a, s);
  return act == kBf16 ? move<kBf16, false>(a, s) : move<kF16, false>(a, s);
}

}  // namespace ea
