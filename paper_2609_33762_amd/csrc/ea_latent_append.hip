// Writing blocks of a latent cache: new tokens' latents as they are and their
// key parts rotated by the position, the queries' parts rotated beside them; or
// tokens of other blocks, their key parts turned from the old position to the
// new one.  fp8 blocks get a scale for their latents and one for their key
// parts, as blocks of keys and values do.
//
// What bounds it is memory.  A workgroup takes a block, its threads 8 elements
// of a token each, side by side over the block.
#include <hip/hip_runtime.h>

#include "ea_kv_blocks.hpp"
#include "ea_kv_device.hpp"

namespace ea {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kLanes;
constexpr int kKeep = 5;  // pieces of 8 elements that a thread keeps in registers

// x of a turned part's piece, with the elements that it turns with: y's in
// place order, or its own neighbours.  c, s: cosines and sines of its pairs.
template <bool INTERLEAVED>
__device__ inline void turn8(float x[8], const float y[8], const float *c, const float *s,
                             bool upper, float sign) {
#pragma clang fp contract(off)
  if constexpr (INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float co = c[i], si = s[i] * sign, a = x[2 * i], b = x[2 * i + 1];
      const float ac = a * co, bs = b * si, bc = b * co, as = a * si;
      x[2 * i] = ac - bs;
      x[2 * i + 1] = bc + as;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float co = c[i], si = s[i] * sign;
      const float xc = x[i] * co, ys = y[i] * si;
      x[i] = upper ? xc + ys : xc - ys;
    }
  }
}

// The turn of piece `rp` of a turned part of `dim` elements at |position| `at`.
template <typename Load>
__device__ inline void turn_piece(float x[8], int rp, const float *rope, int at, float sign,
                                  int dim, bool interleaved, Load partner) {
  const int half = dim >> 1;
  const float *cs = rope + (int64_t)at * dim, *sn = cs + half;
  if (interleaved) {
    turn8<true>(x, nullptr, cs + rp * 4, sn + rp * 4, false, sign);
  } else {
    const int hp = half >> 3;
    const bool upper = rp >= hp;
    const int f = (upper ? rp - hp : rp) * 8;
    float y[8];
    partner(upper ? rp - hp : rp + hp, y);
    turn8<false>(x, y, cs + f, sn + f, upper, sign);
  }
}

// One block's new tokens i0 .. i1-1.  fetch(i, piece, x): piece of token i in
// 32 bits.  Tokens before i0 are older ones that keep their scale, or move to a
// larger one.
template <int ACT, bool FP8, typename Fetch>
__device__ inline void write_block(uint8_t *dst, float *scales, int i0, int i1, int C, int R,
                                   Fetch fetch) {
  constexpr int EB = FP8 ? 1 : 2;
  const int per = (C + R) >> 3, lat = C >> 3, n = (i1 - i0) * per, tid = threadIdx.x;
  __shared__ float most[kWaves][2];
  float x[kKeep][8];
#pragma unroll
  for (int k = 0; k < kKeep; ++k) {
    const int at = tid + k * kThreads;
    if (at < n) fetch(i0 + at / per, at % per, x[k]);
  }
  float scale[2] = {1.f, 1.f};
  if constexpr (FP8) {
    float amax[2] = {0.f, 0.f};
    auto largest = [&](const float y[8], bool turned) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (finite(y[i])) m = fmaxf(m, fabsf(y[i]));
      amax[0] = fmaxf(amax[0], turned ? 0.f : m);
      amax[1] = fmaxf(amax[1], turned ? m : 0.f);
    };
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
      const int at = tid + k * kThreads;
      if (at < n) largest(x[k], at % per >= lat);
    }
    for (int at = tid + kKeep * kThreads; at < n; at += kThreads) {
      float y[8];
      fetch(i0 + at / per, at % per, y);
      largest(y, at % per >= lat);
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      amax[w] = max_wave(amax[w]);
      if ((tid & 63) == 0) most[tid >> 6][w] = amax[w];
    }
    float old[2] = {0.f, 0.f};
    if (i0 > 0) {
      old[0] = scales[0];
      old[1] = scales[1];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float m = most[0][w];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) m = fmaxf(m, most[i][w]);
      scale[w] = fp8_scale(m);
      if (i0 > 0 && old[w] >= scale[w]) scale[w] = old[w];
    }
    if (i0 > 0) {
      const float f[2] = {old[0] * power_inverse(scale[0]), old[1] * power_inverse(scale[1])};
      for (int at = tid; at < i0 * per; at += kThreads) {
        const bool turned = at % per >= lat;
        if (turned ? scale[1] == old[1] : scale[0] == old[0]) continue;
        float y[8];
        u32x2 *q = reinterpret_cast<u32x2 *>(dst + (int64_t)at * 8);
        stored8<ACT, true>(reinterpret_cast<uint8_t *>(q), turned ? f[1] : f[0], y);
        *q = u32x2{fp8_word(y[0], y[1], y[2], y[3]), fp8_word(y[4], y[5], y[6], y[7])};
      }
    }
    if (tid == 0) {
      scales[0] = scale[0];
      scales[1] = scale[1];
    }
  }
  const bool even[2] = {(__float_as_uint(scale[0]) & 0x7fffff) == 0,
                        (__float_as_uint(scale[1]) & 0x7fffff) == 0};
  auto store = [&](int at, const float y[8]) {
    uint8_t *q = dst + ((int64_t)i0 * per + at) * 8 * EB;
    if constexpr (FP8) {
      const bool turned = at % per >= lat;
      const float s = turned ? scale[1] : scale[0], inv = power_inverse(s);
      const bool exact = turned ? even[1] : even[0];
      float z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = exact ? y[i] * inv : y[i] / s;
      *reinterpret_cast<u32x2 *>(q) =
          u32x2{fp8_word(z[0], z[1], z[2], z[3]), fp8_word(z[4], z[5], z[6], z[7])};
    } else {
      *reinterpret_cast<u32x4 *>(q) =
          u32x4{pack_act<ACT>(y[0], y[1]), pack_act<ACT>(y[2], y[3]), pack_act<ACT>(y[4], y[5]),
                pack_act<ACT>(y[6], y[7])};
    }
  };
#pragma unroll
  for (int k = 0; k < kKeep; ++k) {
    const int at = tid + k * kThreads;
    if (at < n) store(at, x[k]);
  }
  for (int at = tid + kKeep * kThreads; at < n; at += kThreads) {
    float y[8];
    fetch(i0 + at / per, at % per, y);
    store(at, y);
  }
}

// The sequence of a row, looked for by all lanes at once (see sequence_of_row).
__device__ inline int32_t sequence_of_row_wave(const BatchRows &b, int32_t row) {
  if (!b.row_start) return row;
  const int lane = threadIdx.x & 63;
  int32_t lo = 0, n = b.n_seqs;
  while (n > 1) {
    const int32_t step = (n + kLanes - 1) / kLanes, at = lo + lane * step;
    const bool before = lane * step < n && b.row_start[at] <= row;
    const int32_t there = max(__popcll(__ballot(before)) - 1, 0) * step;
    lo += there;
    n = min(step, n - there);
  }
  return lo;
}

constexpr int kRowPieces = 4 * kLanes;  // pieces of a row's queries that a wave rotates

template <int ACT, bool FP8>
__global__ __launch_bounds__(kThreads) void append_latent(LatentAppendArgs a, uint32_t blocks) {
  const KvLayer &kv = a.kv;
  const int T = kv.page_tokens, C = a.latent, R = a.turn;
  if (blockIdx.x < blocks) {
    const int s = blockIdx.x / a.pages_most, j = blockIdx.x % a.pages_most;
    const Seq sq = sequence(a.b, s);
    const int start = max(sq.len - sq.rows, 0);  // first new position
    const int p = over_page(kv, start) + j;
    if (p * T >= sq.len) return;
    const int page = a.b.page_table[(int64_t)s * a.b.table_stride + p];
    if ((uint32_t)page >= (uint32_t)kv.num_pages) return;
    const int i0 = max(start - p * T, 0), i1 = min(sq.len - p * T, T);
    // row of the token in slot 0 of this page
    const int64_t row_at = (int64_t)sq.row0 + p * T - (sq.len - sq.rows);
    auto fetch = [&](int i, int piece, float x[8]) {
      const int rp = piece - (C >> 3);
      if (rp < 0) {
        read8<ACT>(a.latents.data + (row_at + i) * a.latents.row_stride + piece * 8, x);
        return;
      }
      const uint16_t *key = a.key.data + (row_at + i) * a.key.row_stride;
      read8<ACT>(key + rp * 8, x);
      if (a.rope)
        turn_piece(x, rp, a.rope, p * T + i, 1.f, R, a.interleaved,
                   [&](int of, float y[8]) { read8<ACT>(key + of * 8, y); });
    };
    write_block<ACT, FP8>(kv.base + page * kv.piece, FP8 ? kv.scales + (int64_t)page * 2 : nullptr,
                          i0, i1, C, R, fetch);
    return;
  }
  // ---- queries
  const int lane = threadIdx.x & 63, per = R >> 3, pieces = a.q_heads * per;
  const int waves = (pieces + kRowPieces - 1) / kRowPieces;
  const uint32_t u = (blockIdx.x - blocks) * kWaves + uniform((int)threadIdx.x >> 6);
  const int row = u / waves;
  if (row >= a.b.n_rows) return;
  const int s = sequence_of_row_wave(a.b, row);
  const Seq sq = sequence(a.b, s);
  const int pos = sq.len - sq.rows + row - sq.row0;
  if (row < sq.row0 || row >= sq.row0 + sq.rows || pos < 0) return;
  const int from = (u % waves) * kRowPieces;
#pragma unroll 4
  for (int at = from + lane; at < min(from + kRowPieces, pieces); at += kLanes) {
    const int h = at / per, rp = at - h * per;
    const uint16_t *src = a.q.data + row * a.q.row_stride + h * a.q.head_stride;
    float x[8];
    read8<ACT>(src + rp * 8, x);
    if (a.rope)
      turn_piece(x, rp, a.rope, pos, 1.f, R, a.interleaved,
                 [&](int of, float y[8]) { read8<ACT>(src + of * 8, y); });
    *reinterpret_cast<u32x4 *>(a.q_out.data + row * a.q_out.row_stride +
                               h * a.q_out.head_stride + rp * 8) =
        u32x4{pack_act<ACT>(x[0], x[1]), pack_act<ACT>(x[2], x[3]), pack_act<ACT>(x[4], x[5]),
              pack_act<ACT>(x[6], x[7])};
  }
}

template <int ACT, bool FP8>
__global__ __launch_bounds__(kThreads) void move_latents(MoveArgs a) {
  constexpr int EB = FP8 ? 1 : 2;
  KvLayer kv = a.kv;
  const int T = kv.page_tokens, C = a.latent, R = a.turn;
  uint32_t u = blockIdx.x;
  const int j = u % a.blocks_most;
  u /= a.blocks_most;
  const int s = u % a.n_seqs, layer = u / a.n_seqs;
  kv.base += layer * a.layer_bytes;
  if (FP8) kv.scales += layer * a.layer_scales;
  const MovedBlock m = moved_block(a, s, j);
  if (m.n <= 0) return;
  const int64_t row_bytes = (int64_t)(C + R) * EB;
  auto fetch = [&](int i, int piece, float x[8]) {
    const MovedToken t = moved_token(a, m, i);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = 0.f;
    if (t.page < 0) return;
    const uint8_t *row = kv.base + t.page * kv.piece + t.slot * row_bytes;
    const int rp = piece - (C >> 3);
    const float scale = FP8 ? kv.scales[(int64_t)t.page * 2 + (rp < 0 ? 0 : 1)] : 1.f;
    stored8<ACT, FP8>(row + piece * 8 * EB, scale, x);
    if (rp >= 0 && a.rope && t.by != 0)
      turn_piece(x, rp, a.rope, abs(t.by), t.by < 0 ? -1.f : 1.f, R, a.interleaved,
                 [&](int of, float y[8]) {
                   stored8<ACT, FP8>(row + (C + of * 8) * EB, scale, y);
                 });
  };
  write_block<ACT, FP8>(kv.base + m.page * kv.piece,
                        FP8 ? kv.scales + (int64_t)m.page * 2 : nullptr, 0, m.n, C, R, fetch);
}

template <int ACT, bool FP8>
hipError_t append(const LatentAppendArgs &a, hipStream_t s) {
  const int64_t blocks = (int64_t)a.b.n_seqs * a.pages_most;
  int64_t grid = blocks;
  if (a.q.data) {
    const int64_t waves = ((int64_t)a.q_heads * (a.turn / 8) + kRowPieces - 1) / kRowPieces;
    grid += (a.b.n_rows * waves + kWaves - 1) / kWaves;
  }
  hipLaunchKernelGGL((append_latent<ACT, FP8>), dim3((unsigned)grid), dim3(kThreads), 0, s, a,
                     (uint32_t)blocks);
  return hipGetLastError();
}

template <int ACT, bool FP8>
hipError_t move(const MoveArgs &a, hipStream_t s) {
  const int64_t grid = (int64_t)a.layers * a.n_seqs * a.blocks_most;
  hipLaunchKernelGGL((move_latents<ACT, FP8>), dim3((unsigned)grid), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append_latent(const LatentAppendArgs &a, int act, int fp8, hipStream_t s) {
  (void)hipGetLastError();
  if (act == kBf16) return fp8 ? append<kBf16, true>(a, s) : append<kBf16, false>(a, s);
  return fp8 ? append<kF16, true>(a, s) : append<kF16, false>(a, s);
}

hipError_t launch_move_latents(const MoveArgs &a, int act, int fp8, hipStream_t s) {
  (void)hipGetLastError();
  if (fp8) return move<kBf16, true>(a, s);
  return act == kBf16 ? move<kBf16, false>(a, s) : move<kF16, false>(a, s);
}

}  // namespace ea
