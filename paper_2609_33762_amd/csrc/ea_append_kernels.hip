// Appending new tokens to the paged cache: keys rotated by their position,
// values as they are, into 16-bit pages or into fp8 pages with a scale for
// each block and head; queries rotated beside them; bounds of the touched
// blocks' keys.
//
// Rotation: (x_i, x_j) -> (x_i cos - x_j sin, x_j cos + x_i sin), each
// product rounded to 32 bits by itself, so that a key is the same wherever
// it is computed.
//
// fp8: the scale of a block and head is the smallest power of two that holds
// its largest magnitude within 448.  e4m3 is a floating format, so a power of
// two costs it nothing, and older tokens of a block whose scale grows are
// requantised without rounding (but for the smallest, subnormal codes).
//
// What bounds it is memory: every input is read once, every output written
// once, apart from a block's older tokens.
#include <hip/hip_runtime.h>

#include "ea_kv_device.hpp"

namespace ea {
namespace {

constexpr int kWaves = 4;

// Lanes side by side on one token's head, 8 elements each.
constexpr int lanes_of(int head_dim) { return head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32; }

template <int ACT>
__device__ inline void read8(const uint16_t *p, float x[8]) {
  const u32x4 v = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = act_to_float<ACT>((uint16_t)(v[i >> 1] >> (16 * (i & 1))));
}

// Elements d0 .. d0+7 of a head, rotated for position `pos`.
template <int ACT>
__device__ inline void rotated8(const uint16_t *head, int d0, const float *rope, int pos, int dim,
                                bool interleaved, float x[8]) {
#pragma clang fp contract(off)
  read8<ACT>(head + d0, x);
  if (d0 >= dim) return;
  const int half = dim >> 1;
  const float *cs = rope + (int64_t)pos * dim, *sn = cs + half;
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (d0 + 2 * i >= dim) break;
      const float co = cs[(d0 >> 1) + i], si = sn[(d0 >> 1) + i];
      const float a = x[2 * i], b = x[2 * i + 1];
      const float ac = a * co, bs = b * si, bc = b * co, as = a * si;
      x[2 * i] = ac - bs;
      x[2 * i + 1] = bc + as;
    }
  } else if ((half & 7) == 0) {  // the partners are 8 neighbours too
    const bool upper = d0 >= half;
    float y[8];
    read8<ACT>(head + (upper ? d0 - half : d0 + half), y);
    const int f0 = upper ? d0 - half : d0;
    const f32x4 c0 = *reinterpret_cast<const f32x4 *>(cs + f0);
    const f32x4 c1 = *reinterpret_cast<const f32x4 *>(cs + f0 + 4);
    const f32x4 s0 = *reinterpret_cast<const f32x4 *>(sn + f0);
    const f32x4 s1 = *reinterpret_cast<const f32x4 *>(sn + f0 + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float co = i < 4 ? c0[i & 3] : c1[i & 3], si = i < 4 ? s0[i & 3] : s1[i & 3];
      const float xc = x[i] * co, ys = y[i] * si;
      x[i] = upper ? xc + ys : xc - ys;
    }
  } else {
    for (int i = 0; i < 8; ++i) {
      const int d = d0 + i;
      if (d >= dim) break;
      const bool upper = d >= half;
      const int f = upper ? d - half : d;
      const float y = act_to_float<ACT>(head[upper ? d - half : d + half]);
      const float xc = x[i] * cs[f], ys = y * sn[f];
      x[i] = upper ? xc + ys : xc - ys;
    }
  }
}

__device__ inline float max_wave(float v) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// Four fp8 codes from four values and back.
__device__ inline uint32_t fp8_word(float a, float b, float c, float d) {
  uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ inline void fp8_values(uint32_t w, float x[4]) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
  const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  x[0] = a[0];
  x[1] = a[1];
  x[2] = b[0];
  x[3] = b[1];
}

// Elements d0 .. d0+7 of a stored token as values.
template <int ACT, bool FP8>
__device__ inline void stored8(const uint8_t *p, float scale, float x[8]) {
  if constexpr (FP8) {
    const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
    fp8_values(w[0], x);
    fp8_values(w[1], x + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= scale;
  } else {
    read8<ACT>(reinterpret_cast<const uint16_t *>(p), x);
  }
}

// Bounds of a block's keys as whole numbers: lowest rounded down, highest
// rounded up, in units of a power of two that holds them within 127.  Lanes
// hold 8 elements each of every (64 / LD)-th token.  Values that are not
// finite do not set the unit; an infinity is the largest whole number.
template <int LD>
__device__ inline void write_bounds(const KvLayer &kv, int page, int h, int lane, float lo[8],
                                    float hi[8]) {
  const int D = kv.head_dim, d0 = (lane % LD) * 8;
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    for (int d = LD; d < kLanes; d <<= 1) {
      lo[i] = fminf(lo[i], __shfl_xor(lo[i], d));
      hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], d));
    }
    if (d0 < D && finite(lo[i])) amax = fmaxf(amax, fabsf(lo[i]));
    if (d0 < D && finite(hi[i])) amax = fmaxf(amax, fabsf(hi[i]));
  }
  const float s = int8_scale(max_wave(amax)), inv = power_inverse(s);
  if (lane < LD && d0 < D) {
    u32x2 wl = {0, 0}, wh = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int l = (int)fmaxf(fminf(floorf(lo[i] * inv), 127.f), -127.f);
      const int u = (int)fmaxf(fminf(ceilf(hi[i] * inv), 127.f), -127.f);
      wl[i >> 2] |= (uint32_t)(uint8_t)l << (8 * (i & 3));
      wh[i >> 2] |= (uint32_t)(uint8_t)u << (8 * (i & 3));
    }
    int8_t *p = kv.bounds + ((int64_t)page * 2 * kv.heads + h) * D + d0;
    *reinterpret_cast<u32x2 *>(p) = wl;
    *reinterpret_cast<u32x2 *>(p + (int64_t)kv.heads * D) = wh;
  }
  if (lane == 0) kv.bound_scales[(int64_t)page * kv.heads + h] = s;
}

// One wave: the new tokens of one block, for one KV head, keys or values.
template <int ACT, bool FP8, int LD>
__device__ inline void append_block(const AppendArgs &a, uint32_t u, int lane) {
  const KvLayer &kv = a.kv;
  constexpr int EB = FP8 ? 1 : 2, TW = kLanes / LD;  // tokens of a pass
  const int H = kv.heads, D = kv.head_dim, T = kv.page_tokens;
  const bool value = u & 1;
  u >>= 1;
  const int h = u % H;
  u /= H;
  const int j = u % a.pages_most, s = u / a.pages_most;
  const Seq sq = sequence(a.b, s);
  const int start = max(sq.len - sq.rows, 0);  // first new position
  const int p = over_page(kv, start) + j;
  if (p * T >= sq.len) return;
  const int page = a.b.page_table[(int64_t)s * a.b.table_stride + p];
  if ((uint32_t)page >= (uint32_t)kv.num_pages) return;
  const int i0 = max(start - p * T, 0), i1 = min(sq.len - p * T, T);
  const int64_t token_bytes = (int64_t)H * D * EB;
  const int d0 = (lane % LD) * 8, t0 = lane / LD;
  const bool in = d0 < D;
  uint8_t *dst = kv.base + page * kv.piece + (value ? kv.piece >> 1 : 0) +
                 ((int64_t)h * D + (in ? d0 : 0)) * EB;
  const HeadRows &src = value ? a.v : a.k;
  // row of the token in slot t of this page
  const int64_t row_at = (int64_t)sq.row0 + p * T - (sq.len - sq.rows);
  const uint16_t *head = src.data + row_at * src.row_stride + (int64_t)h * src.head_stride;
  const bool turn = !value && a.rope;
  auto fetch = [&](int t, float x[8]) {
    if (turn) rotated8<ACT>(head + t * src.row_stride, d0, a.rope, p * T + t, a.rope_dim,
                            a.interleaved, x);
    else read8<ACT>(head + t * src.row_stride + d0, x);
  };
  float scale = 1.f, inv = 1.f;
  bool even = true;  // a power of two, as this kernel writes them
  if constexpr (FP8) {
    float amax = 0.f;
    for (int t = i0 + t0; t < i1; t += TW) {
      if (!in) continue;
      float x[8];
      fetch(t, x);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (finite(x[i])) amax = fmaxf(amax, fabsf(x[i]));
    }
    scale = fp8_scale(max_wave(amax));
    float *sp = kv.scales + (int64_t)page * kv.scale_page + (value ? kv.scale_kv : 0) +
                h * kv.scale_head;
    if (i0 > 0) {  // older tokens keep their scale or move to the larger one
      const float old = *sp;
      if (old >= scale) {
        scale = old;
      } else {
        const float f = old * power_inverse(scale);
        for (int t = t0; t < i0; t += TW) {
          if (!in) continue;
          float x[8];
          stored8<ACT, true>(dst + t * token_bytes, f, x);
          *reinterpret_cast<u32x2 *>(dst + t * token_bytes) =
              u32x2{fp8_word(x[0], x[1], x[2], x[3]), fp8_word(x[4], x[5], x[6], x[7])};
        }
      }
    }
    even = (__float_as_uint(scale) & 0x7fffff) == 0;
    inv = power_inverse(scale);
    if (lane == 0) *sp = scale;
  }
  const bool bounds = !value && kv.bounds;
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo[i] = __builtin_inff();
    hi[i] = kNegInf;
  }
  auto hold = [&](const float x[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[i] = fminf(lo[i], x[i]);
      hi[i] = fmaxf(hi[i], x[i]);
    }
  };
  for (int t = i0 + t0; t < i1; t += TW) {
    if (!in) continue;
    float x[8];
    fetch(t, x);
    if constexpr (FP8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = even ? x[i] * inv : x[i] / scale;
      const u32x2 w = {fp8_word(x[0], x[1], x[2], x[3]), fp8_word(x[4], x[5], x[6], x[7])};
      *reinterpret_cast<u32x2 *>(dst + t * token_bytes) = w;
      if (bounds) {
        fp8_values(w[0], x);
        fp8_values(w[1], x + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= scale;
        hold(x);
      }
    } else {
      const u32x4 w = {pack_act<ACT>(x[0], x[1]), pack_act<ACT>(x[2], x[3]),
                       pack_act<ACT>(x[4], x[5]), pack_act<ACT>(x[6], x[7])};
      *reinterpret_cast<u32x4 *>(dst + t * token_bytes) = w;
      if (bounds) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[i] = act_to_float<ACT>((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
        hold(x);
      }
    }
  }
  if (bounds) {  // the block's older tokens count too; this lane wrote them last
    for (int t = t0; t < i0; t += TW) {
      if (!in) continue;
      float x[8];
      stored8<ACT, FP8>(dst + t * token_bytes, scale, x);
      hold(x);
    }
    write_bounds<LD>(kv, page, h, lane, lo, hi);
  }
}

constexpr int kQueryHeads = 16;  // heads of a row one wave rotates

template <int ACT, int LD>
__device__ inline void rotate_queries(const AppendArgs &a, uint32_t u, int lane) {
  constexpr int HW = kLanes / LD;
  const int D = a.kv.head_dim, groups = (a.q_heads + kQueryHeads - 1) / kQueryHeads;
  const int h0 = (u % groups) * kQueryHeads, row = u / groups;
  if (row >= a.b.n_rows) return;
  const int s = sequence_of_row(a.b, row);
  const Seq sq = sequence(a.b, s);
  const int pos = sq.len - sq.rows + row - sq.row0;
  if (row < sq.row0 || row >= sq.row0 + sq.rows || pos < 0) return;
  const int d0 = (lane % LD) * 8;
  if (d0 >= D) return;
#pragma unroll
  for (int i = 0; i < kQueryHeads; i += HW) {
    const int h = h0 + i + lane / LD;
    if (h >= a.q_heads) break;
    float x[8];
    const uint16_t *src = a.q.data + row * a.q.row_stride + h * a.q.head_stride;
    if (a.rope) rotated8<ACT>(src, d0, a.rope, pos, a.rope_dim, a.interleaved, x);
    else read8<ACT>(src + d0, x);
    *reinterpret_cast<u32x4 *>(a.q_out.data + row * a.q_out.row_stride +
                               h * a.q_out.head_stride + d0) =
        u32x4{pack_act<ACT>(x[0], x[1]), pack_act<ACT>(x[2], x[3]), pack_act<ACT>(x[4], x[5]),
              pack_act<ACT>(x[6], x[7])};
  }
}

template <int ACT, bool FP8, int LD>
__global__ __launch_bounds__(kWaves *kLanes) void append_kv(AppendArgs a, uint32_t block_units,
                                                            uint32_t units) {
  const int lane = threadIdx.x & 63;
  const uint32_t u = blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  if (u >= units) return;
  if (u < block_units) append_block<ACT, FP8, LD>(a, u, lane);
  else rotate_queries<ACT, LD>(a, u - block_units, lane);
}

// Bounds of whole blocks from what is stored in them.
template <int ACT, bool FP8, int LD>
__global__ __launch_bounds__(kWaves *kLanes) void bound_blocks(KvLayer kv, const int32_t *pages,
                                                               int64_t units, int64_t layer_bytes,
                                                               int64_t layer_scales, int32_t n) {
  constexpr int EB = FP8 ? 1 : 2;
  const int lane = threadIdx.x & 63;
  int64_t u = (int64_t)blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  if (u >= units) return;
  const int H = kv.heads, D = kv.head_dim;
  const int h = u % H;
  u /= H;
  const int page = pages[u % n];
  if ((uint32_t)page >= (uint32_t)kv.num_pages) return;
  const int64_t l = u / n;
  kv.base += l * layer_bytes;
  kv.bounds += l * kv.num_pages * 2 * H * D;
  kv.bound_scales += l * kv.num_pages * H;
  float scale = 1.f;
  if (FP8)
    scale = kv.scales[l * layer_scales + (int64_t)page * kv.scale_page + h * kv.scale_head];
  const int d0 = (lane % LD) * 8;
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo[i] = __builtin_inff();
    hi[i] = kNegInf;
  }
  if (d0 < D)
    for (int t = lane / LD; t < kv.page_tokens; t += kLanes / LD) {
      float x[8];
      stored8<ACT, FP8>(kv.base + page * kv.piece + ((int64_t)(t * H + h) * D + d0) * EB, scale,
                        x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        lo[i] = fminf(lo[i], x[i]);
        hi[i] = fmaxf(hi[i], x[i]);
      }
    }
  write_bounds<LD>(kv, page, h, lane, lo, hi);
}

template <int ACT, bool FP8>
hipError_t append(const AppendArgs &a, hipStream_t s) {
  const int64_t blocks = (int64_t)a.b.n_seqs * a.pages_most * a.kv.heads * 2;
  const int64_t units =
      blocks + (a.q.data ? (int64_t)a.b.n_rows * ((a.q_heads + kQueryHeads - 1) / kQueryHeads) : 0);
  const dim3 grid((unsigned)((units + kWaves - 1) / kWaves)), block(kWaves * kLanes);
  const uint32_t nb = (uint32_t)blocks, nu = (uint32_t)units;
  switch (lanes_of(a.kv.head_dim)) {
    case 8: hipLaunchKernelGGL((append_kv<ACT, FP8, 8>), grid, block, 0, s, a, nb, nu); break;
    case 16: hipLaunchKernelGGL((append_kv<ACT, FP8, 16>), grid, block, 0, s, a, nb, nu); break;
    default: hipLaunchKernelGGL((append_kv<ACT, FP8, 32>), grid, block, 0, s, a, nb, nu);
  }
  return hipGetLastError();
}

template <int ACT, bool FP8>
hipError_t bounds(const KvLayer &kv, int32_t layers, int64_t lb, int64_t ls, const int32_t *pages,
                  int32_t n, hipStream_t s) {
  const int64_t units = (int64_t)layers * n * kv.heads;
  const dim3 grid((unsigned)((units + kWaves - 1) / kWaves)), block(kWaves * kLanes);
  switch (lanes_of(kv.head_dim)) {
    case 8:
      hipLaunchKernelGGL((bound_blocks<ACT, FP8, 8>), grid, block, 0, s, kv, pages, units, lb, ls,
                         n);
      break;
    case 16:
      hipLaunchKernelGGL((bound_blocks<ACT, FP8, 16>), grid, block, 0, s, kv, pages, units, lb,
                         ls, n);
      break;
    default:
      hipLaunchKernelGGL((bound_blocks<ACT, FP8, 32>), grid, block, 0, s, kv, pages, units, lb,
                         ls, n);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, int act, hipStream_t s) {
  (void)hipGetLastError();
  if (act == kBf16) return a.fp8 ? append<kBf16, true>(a, s) : append<kBf16, false>(a, s);
  return a.fp8 ? append<kF16, true>(a, s) : append<kF16, false>(a, s);
}

hipError_t launch_bounds(const KvLayer &kv, int act, int fp8, int32_t layers, int64_t layer_bytes,
                         int64_t layer_scales, const int32_t *pages, int32_t n, hipStream_t s) {
  (void)hipGetLastError();
  if (fp8) return bounds<kBf16, true>(kv, layers, layer_bytes, layer_scales, pages, n, s);
  if (act == kBf16)
    return bounds<kBf16, false>(kv, layers, layer_bytes, layer_scales, pages, n, s);
  return bounds<kF16, false>(kv, layers, layer_bytes, layer_scales, pages, n, s);
}

}  // namespace ea
