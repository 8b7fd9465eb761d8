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
// once, apart from a block's older tokens.  A wave takes a block's head, keys or
// values, so its scale and bounds need no other wave; queries are units of
// their own.  32,000 new tokens into 16-bit pages, 671 MB in all, take 128 us
// (5.2 TB/s), ragged fp8 chunks of 241 MB 64 us (3.8 TB/s); 64 single tokens
// into fp8 blocks take 9 us, a block's tokens read, turned and written one
// after another.
#include <hip/hip_runtime.h>

#include "ea_kv_blocks.hpp"
#include "ea_kv_device.hpp"

namespace ea {
namespace {

constexpr int kWaves = 4;

// A lane's elements of a head, rotated for position `pos` where `rope` is not
// null.  HALVES: the rotation, if any, pairs whole pieces; the other ways of
// pairing need registers that this one leaves to more waves.
template <int ACT, bool HALVES>
__device__ inline void rotated(const uint16_t *head, const Place &p, const float *rope, int pos,
                               int dim, bool interleaved, const Angles &an, float x[16]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    if (p.in[n]) {
      read8<ACT>(head + p.d[n], x + n * 8);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[n * 8 + i] = 0.f;
    }
  }
  if (!rope) return;
  if (p.paired) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float co = an.c[i >> 2][i & 3], si = an.s[i >> 2][i & 3], a = x[i], b = x[8 + i];
      const float ac = a * co, bs = b * si, bc = b * co, as = a * si;
      x[i] = ac - bs;
      x[8 + i] = bc + as;
    }
    return;
  }
  if constexpr (HALVES) return;  // past what turns
  const int half = dim >> 1;
  const float *cs = rope + (int64_t)pos * dim, *sn = cs + half;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    if (!p.in[n] || p.d[n] >= dim) continue;
    if (interleaved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int f = (p.d[n] >> 1) + i;
        if (f >= half) break;
        const float a = x[n * 8 + 2 * i], b = x[n * 8 + 2 * i + 1];
        const float ac = a * cs[f], bs = b * sn[f], bc = b * cs[f], as = a * sn[f];
        x[n * 8 + 2 * i] = ac - bs;
        x[n * 8 + 2 * i + 1] = bc + as;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = p.d[n] + i;
        if (d >= dim) break;
        const bool upper = d >= half;
        const int f = upper ? d - half : d;
        const float y = act_to_float<ACT>(head[upper ? d - half : d + half]);
        const float xc = x[n * 8 + i] * cs[f], ys = y * sn[f];
        x[n * 8 + i] = upper ? xc + ys : xc - ys;
      }
    }
  }
}

// One wave: the new tokens of one block, for one KV head, keys or values.
template <int ACT, bool FP8, int LP, bool HALVES>
__device__ inline void append_block(const AppendArgs &a, uint32_t u, int lane) {
  const KvLayer &kv = a.kv;
  constexpr int EB = FP8 ? 1 : 2, TW = kLanes / LP;  // tokens of a pass
  constexpr int KEEP = 2;  // passes whose tokens stay in registers
  const int H = kv.heads, D = kv.head_dim, T = kv.page_tokens;
  const bool value = u & 1;
  u >>= 1;
  const int h = u % H;
  u /= H;
  const int j = u % a.pages_most, s = u / a.pages_most;
  const Seq sq = sequence(a.b, s);
  // (nothing of a sequence without rows is read or written: its length and table
  // may be those of an earlier step, its pages another sequence's by now)
  if (sq.rows == 0) return;
  const int start = max(sq.len - sq.rows, 0);  // first new position
  const int p = over_page(kv, start) + j;
  if (p * T >= sq.len) return;
  const int page = a.b.page_table[(int64_t)s * a.b.table_stride + p];
  if ((uint32_t)page >= (uint32_t)kv.num_pages) return;
  const int i0 = max(start - p * T, 0), i1 = min(sq.len - p * T, T);
  const int64_t token_bytes = (int64_t)H * D * EB;
  const int t0 = lane / LP;
  const float *rope = value ? nullptr : a.rope;
  const Place at = place_of(lane % LP, D, rope != nullptr, a.rope_dim, a.interleaved);
  uint8_t *dst = kv.base + page * kv.piece + (value ? kv.piece >> 1 : 0) + (int64_t)h * D * EB;
  const HeadRows &src = value ? a.v : a.k;
  // row of the token in slot t of this page
  const int64_t row_at = (int64_t)sq.row0 + p * T - (sq.len - sq.rows);
  const uint16_t *head = src.data + row_at * src.row_stride + (int64_t)h * src.head_stride;
  auto fetch = [&](int t, float x[16]) {
    Angles an = {};
    if (rope) an = angles_of(rope, p * T + t, a.rope_dim, at);
    rotated<ACT, HALVES>(head + t * src.row_stride, at, rope, p * T + t, a.rope_dim,
                         a.interleaved, an, x);
  };
  // the first passes' tokens; a block of more is read again below
  float x[KEEP][16];
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (i0 + t0 + k * TW < i1) fetch(i0 + t0 + k * TW, x[k]);
  float scale = 1.f, inv = 1.f;
  bool even = true;  // a power of two, as this kernel writes them
  if constexpr (FP8) {
    float amax = 0.f;
    auto largest = [&](const float y[16]) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (finite(y[i])) amax = fmaxf(amax, fabsf(y[i]));
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
      if (i0 + t0 + k * TW < i1) largest(x[k]);
    for (int t = i0 + t0 + KEEP * TW; t < i1; t += TW) {
      float y[16];
      fetch(t, y);
      largest(y);
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
        for (int t = t0; t < i0; t += TW)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            if (!at.in[n]) continue;
            float y[8];
            uint8_t *q = dst + t * token_bytes + at.d[n] * EB;
            stored8<ACT, true>(q, f, y);
            *reinterpret_cast<u32x2 *>(q) =
                u32x2{fp8_word(y[0], y[1], y[2], y[3]), fp8_word(y[4], y[5], y[6], y[7])};
          }
      }
    }
    even = (__float_as_uint(scale) & 0x7fffff) == 0;
    inv = power_inverse(scale);
    if (lane == 0) *sp = scale;
  }
  const bool bounds = !value && kv.bounds;
  float lo[16], hi[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    lo[i] = __builtin_inff();
    hi[i] = kNegInf;
  }
  auto hold = [&](int n, const float y[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[n * 8 + i] = fminf(lo[n * 8 + i], y[i]);
      hi[n * 8 + i] = fmaxf(hi[n * 8 + i], y[i]);
    }
  };
  auto store = [&](int t, const float y[16]) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      if (!at.in[n]) continue;
      uint8_t *q = dst + t * token_bytes + at.d[n] * EB;
      float z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = y[n * 8 + i];
      if constexpr (FP8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = even ? z[i] * inv : z[i] / scale;
        const u32x2 w = {fp8_word(z[0], z[1], z[2], z[3]), fp8_word(z[4], z[5], z[6], z[7])};
        *reinterpret_cast<u32x2 *>(q) = w;
        if (bounds) {
          fp8_values(w[0], z);
          fp8_values(w[1], z + 4);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] *= scale;
          hold(n, z);
        }
      } else {
        const u32x4 w = {pack_act<ACT>(z[0], z[1]), pack_act<ACT>(z[2], z[3]),
                         pack_act<ACT>(z[4], z[5]), pack_act<ACT>(z[6], z[7])};
        *reinterpret_cast<u32x4 *>(q) = w;
        if (bounds) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            z[i] = act_to_float<ACT>((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
          hold(n, z);
        }
      }
    }
  };
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (i0 + t0 + k * TW < i1) store(i0 + t0 + k * TW, x[k]);
  for (int t = i0 + t0 + KEEP * TW; t < i1; t += TW) {
    float y[16];
    fetch(t, y);
    store(t, y);
  }
  if (bounds) {  // the block's older tokens count too; this lane wrote them last
    for (int t = t0; t < i0; t += TW)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        if (!at.in[n]) continue;
        float y[8];
        stored8<ACT, FP8>(dst + t * token_bytes + at.d[n] * EB, scale, y);
        hold(n, y);
      }
    write_bounds<LP>(kv, page, h, lane, at, lo, hi);
  }
}

constexpr int kQueryHeads = 16;  // heads of a row one wave rotates

template <int ACT, int LP, bool HALVES>
__device__ inline void rotate_queries(const AppendArgs &a, uint32_t u, int lane) {
  constexpr int HW = kLanes / LP;
  const int D = a.kv.head_dim, groups = (a.q_heads + kQueryHeads - 1) / kQueryHeads;
  const int h0 = (u % groups) * kQueryHeads, row = u / groups;
  if (row >= a.b.n_rows) return;
  const int s = sequence_of_row(a.b, row);
  const Seq sq = sequence(a.b, s);
  const int pos = sq.len - sq.rows + row - sq.row0;
  if (row < sq.row0 || row >= sq.row0 + sq.rows || pos < 0) return;
  const Place at = place_of(lane % LP, D, a.rope != nullptr, a.rope_dim, a.interleaved);
  Angles an = {};
  if (a.rope) an = angles_of(a.rope, pos, a.rope_dim, at);
  const uint16_t *src = a.q.data + row * a.q.row_stride;
  uint16_t *dst = a.q_out.data + row * a.q_out.row_stride;
#pragma unroll
  for (int i = 0; i < kQueryHeads; i += HW) {
    const int h = h0 + i + lane / LP;
    if (h >= a.q_heads) break;
    float x[16];
    rotated<ACT, HALVES>(src + h * a.q.head_stride, at, a.rope, pos, a.rope_dim, a.interleaved,
                         an, x);
#pragma unroll
    for (int n = 0; n < 2; ++n)
      if (at.in[n])
        *reinterpret_cast<u32x4 *>(dst + h * a.q_out.head_stride + at.d[n]) =
            u32x4{pack_act<ACT>(x[n * 8], x[n * 8 + 1]), pack_act<ACT>(x[n * 8 + 2], x[n * 8 + 3]),
                  pack_act<ACT>(x[n * 8 + 4], x[n * 8 + 5]),
                  pack_act<ACT>(x[n * 8 + 6], x[n * 8 + 7])};
  }
}

template <int ACT, bool FP8, int LP, bool HALVES>
__global__ __launch_bounds__(kWaves *kLanes) void append_kv(AppendArgs a, uint32_t block_units,
                                                            uint32_t units) {
  const int lane = threadIdx.x & 63;
  const uint32_t u = blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  if (u >= units) return;
  if (u < block_units) append_block<ACT, FP8, LP, HALVES>(a, u, lane);
  else rotate_queries<ACT, LP, HALVES>(a, u - block_units, lane);
}

// Bounds of whole blocks from what is stored in them.
template <int ACT, bool FP8, int LP>
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
  const Place at = place_of(lane % LP, D, false, 0, false);
  float lo[16], hi[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    lo[i] = __builtin_inff();
    hi[i] = kNegInf;
  }
  for (int t = lane / LP; t < kv.page_tokens; t += kLanes / LP)
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      if (!at.in[n]) continue;
      float x[8];
      stored8<ACT, FP8>(kv.base + page * kv.piece + ((int64_t)(t * H + h) * D + at.d[n]) * EB,
                        scale, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        lo[n * 8 + i] = fminf(lo[n * 8 + i], x[i]);
        hi[n * 8 + i] = fmaxf(hi[n * 8 + i], x[i]);
      }
    }
  write_bounds<LP>(kv, page, h, lane, at, lo, hi);
}

template <int ACT, bool FP8, int LP>
void append_as(const AppendArgs &a, dim3 grid, uint32_t blocks, uint32_t units, hipStream_t s) {
  const dim3 block(kWaves * kLanes);
  if (!a.rope || (!a.interleaved && a.rope_dim % 16 == 0))
    hipLaunchKernelGGL((append_kv<ACT, FP8, LP, true>), grid, block, 0, s, a, blocks, units);
  else
    hipLaunchKernelGGL((append_kv<ACT, FP8, LP, false>), grid, block, 0, s, a, blocks, units);
}

template <int ACT, bool FP8>
hipError_t append(const AppendArgs &a, hipStream_t s) {
  const int64_t blocks = (int64_t)a.b.n_seqs * a.pages_most * a.kv.heads * 2;
  const int64_t units =
      blocks + (a.q.data ? (int64_t)a.b.n_rows * ((a.q_heads + kQueryHeads - 1) / kQueryHeads) : 0);
  const dim3 grid((unsigned)((units + kWaves - 1) / kWaves));
  const uint32_t nb = (uint32_t)blocks, nu = (uint32_t)units;
  switch (lanes_of(a.kv.head_dim)) {
    case 4: append_as<ACT, FP8, 4>(a, grid, nb, nu, s); break;
    case 8: append_as<ACT, FP8, 8>(a, grid, nb, nu, s); break;
    default: append_as<ACT, FP8, 16>(a, grid, nb, nu, s);
  }
  return hipGetLastError();
}

template <int ACT, bool FP8>
hipError_t bounds(const KvLayer &kv, int32_t layers, int64_t lb, int64_t ls, const int32_t *pages,
                  int32_t n, hipStream_t s) {
  const int64_t units = (int64_t)layers * n * kv.heads;
  const dim3 grid((unsigned)((units + kWaves - 1) / kWaves)), block(kWaves * kLanes);
  switch (lanes_of(kv.head_dim)) {
    case 4:
      hipLaunchKernelGGL((bound_blocks<ACT, FP8, 4>), grid, block, 0, s, kv, pages, units, lb, ls,
                         n);
      break;
    case 8:
      hipLaunchKernelGGL((bound_blocks<ACT, FP8, 8>), grid, block, 0, s, kv, pages, units, lb,
                         ls, n);
      break;
    default:
      hipLaunchKernelGGL((bound_blocks<ACT, FP8, 16>), grid, block, 0, s, kv, pages, units, lb,
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
