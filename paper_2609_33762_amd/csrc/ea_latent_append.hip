// Writing blocks of a latent cache: new tokens' latents as they are and their
// key parts rotated by the position, the queries' parts rotated beside them; or
// tokens of other blocks, their key parts turned from the old position to the
// new one.  fp8 blocks get a scale for their latents and one for their key
// parts, as blocks of keys and values do.
//
// What bounds it is memory.  A workgroup takes a block, its threads 8 elements
// of a token each, side by side over the block, and keeps them in registers between
// the search for the largest value and the rounding, so that each is read once.
// Queries go by waves of the same launch.  Measured: 5 ragged pieces of prompts, fp8,
// 54 MB: 15-17 us (3.3 TB/s); 4 tokens: 3.7 us.
// Moved 16-bit latents, 953 MB: 205 us (4.6 TB/s); with latents unpacked and packed
// again as their turned parts are 277.
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

// Heads of a row's queries that a wave rotates, and rotates at once: whole ones, as
// q_out may be q and a head's halves turn together.
__host__ __device__ inline int heads_at_once(int per) { return kLanes / per; }
__host__ __device__ inline int heads_of_wave(int per) { return 4 * heads_at_once(per); }

template <int ACT, bool FP8>
__global__ __launch_bounds__(kThreads) void append_latent(LatentAppendArgs a, uint32_t blocks) {
  const KvLayer &kv = a.kv;
  const int T = kv.page_tokens, C = a.latent, R = a.turn;
  if (blockIdx.x < blocks) {
    const int s = blockIdx.x / a.pages_most, j = blockIdx.x % a.pages_most;
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
  const int lane = threadIdx.x & 63, per = R >> 3, once = heads_at_once(per);
  const int wave_heads = heads_of_wave(per), waves = (a.q_heads + wave_heads - 1) / wave_heads;
  const uint32_t u = (blockIdx.x - blocks) * kWaves + uniform((int)threadIdx.x >> 6);
  const int row = u / waves;
  if (row >= a.b.n_rows) return;
  const int s = sequence_of_row_wave(a.b, row);
  const Seq sq = sequence(a.b, s);
  const int pos = sq.len - sq.rows + row - sq.row0;
  if (row < sq.row0 || row >= sq.row0 + sq.rows || pos < 0) return;
  const int h0 = lane / per, rp = lane - h0 * per, from = (u % waves) * wave_heads;
  const int to = min(from + wave_heads, a.q_heads);
  if (h0 >= once) return;
#pragma unroll 4
  for (int h = from + h0; h < to; h += once) {
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

// Moved rows: a workgroup takes up to 16 tokens (fp8: a block, 16 tokens at a
// time) through some layers.  A thread has 16-byte pieces of their latents, which
// only fp8 looks into, and one piece of 8 turned elements, with the piece that
// it turns with and its angles, which serve all layers.
template <int ACT, bool FP8>
__global__ __launch_bounds__(kThreads) void move_latents(MoveArgs a) {
  constexpr int EB = FP8 ? 1 : 2, PER = 16 / EB;  // elements of a piece
  constexpr int KEEP = 16 * kMaxLatent / PER / kThreads;
  constexpr int W = FP8 ? 2 : 4;                  // words of 8 elements
  __shared__ float most[2][kWaves][2];
  const int T = a.kv.page_tokens, C = a.latent, R = a.turn, tid = threadIdx.x;
  const uint32_t row_bytes = (C + R) * EB;
  uint32_t u = blockIdx.x;
  const int j = u % a.blocks_most;
  u /= a.blocks_most;
  const int s = u % a.n_seqs, layer0 = u / a.n_seqs * a.layers_wave;
  const int layer1 = min(layer0 + a.layers_wave, a.layers);
  // fp8: the block's tokens; else 16 of the sequence, whose blocks they are in
  // is looked up for each
  MovedBlock m;
  if constexpr (FP8) m = moved_block(a, s, j);
  else m = moved_run(a, s, j * 16, 16);
  if (m.n <= 0) return;
  const int32_t *dst_table = a.dst_table + (int64_t)s * a.dst_stride;
  const int groups = FP8 ? (m.n + 15) / 16 : 1;

  const int lat = C / PER, trn = R >> 3, half = trn >> 1;  // pieces of a token
  // place in the layer that a piece comes from (-1: zeros) and goes to (-1: nowhere)
  int64_t src[KEEP], dst[KEEP], tsrc, tdst;
  uint32_t src_page[KEEP], tsrc_page;
  int tby = 0, apart = 0;  // the turn, and the other piece's distance in bytes
  f32x4 c[2], sn[2];
  bool upper = false;
  auto to_of = [&](int i) -> int64_t {  // row that token i goes to
    if constexpr (FP8) return m.page * a.kv.piece + (int64_t)i * row_bytes;
    const int at = j * 16 + i, e = over_page(a.kv, at);
    const int page = dst_table[e];
    if ((uint32_t)page >= (uint32_t)a.kv.num_pages) return -1;
    return page * a.kv.piece + (int64_t)(at - e * T) * row_bytes;
  };
  auto places = [&](int group) {
    const int n = min(m.n - group * 16, 16);
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
      const int at = tid + k * kThreads, i = at / lat, piece = at - i * lat;
      src[k] = dst[k] = -1;
      src_page[k] = 0;
      if (i >= n) continue;
      const MovedToken t = moved_token(a, m, group * 16 + i);
      const int64_t to = to_of(group * 16 + i);
      if (to >= 0) dst[k] = to + piece * 16;
      if (t.page < 0) continue;
      src_page[k] = t.page;
      src[k] = t.page * a.kv.piece + (int64_t)t.slot * row_bytes + piece * 16;
    }
    tsrc = tdst = -1;
    tsrc_page = 0;
    const int i = tid / trn, piece = tid - i * trn;
    if (i >= n) return;
    const MovedToken t = moved_token(a, m, group * 16 + i);
    const int64_t to = to_of(group * 16 + i);
    if (to >= 0) tdst = to + C * EB + piece * 8 * EB;
    if (t.page < 0) return;
    tsrc_page = t.page;
    tsrc = t.page * a.kv.piece + (int64_t)t.slot * row_bytes + C * EB + piece * 8 * EB;
    tby = t.by;
    if (tby == 0) return;
    upper = piece >= half;
    apart = a.interleaved ? 0 : (upper ? -half : half) * 8 * EB;
    const float *cs = a.rope + (int64_t)abs(tby) * R + (a.interleaved ? piece * 4
                                                        : (upper ? piece - half : piece) * 8);
    const float *ss = cs + (R >> 1);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int more = a.interleaved ? 0 : q * 4;  // four pairs then
      c[q] = *reinterpret_cast<const f32x4 *>(cs + more);
      sn[q] = *reinterpret_cast<const f32x4 *>(ss + more);
      if (tby < 0) sn[q] = -sn[q];
    }
  };
  struct Raw {
    u32x4 lat[KEEP];
    float lat_scale[KEEP], turn_scale;
    uint32_t own[W], other[W];
  };
  auto load8 = [&](const uint8_t *p, uint32_t w[W]) {
    if constexpr (FP8) {
      const u32x2 v = *reinterpret_cast<const u32x2 *>(p);
      w[0] = v[0];
      w[1] = v[1];
    } else {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i];
    }
  };
  auto load = [&](int layer) {
    Raw r = {};
    const uint8_t *base = a.kv.base + layer * a.layer_bytes;
    const float *scales = FP8 ? a.kv.scales + layer * a.layer_scales : nullptr;
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
      r.lat_scale[k] = 0.f;
      if (src[k] >= 0) {
        r.lat[k] = *reinterpret_cast<const u32x4 *>(base + src[k]);
        if (FP8) r.lat_scale[k] = scales[(int64_t)src_page[k] * 2];
      }
    }
    r.turn_scale = 0.f;
    if (tsrc >= 0) {
      load8(base + tsrc, r.own);
      if (tby != 0) load8(base + tsrc + apart, r.other);
      if (FP8) r.turn_scale = scales[(int64_t)tsrc_page * 2 + 1];
    }
    return r;
  };
  auto values8 = [&](const uint32_t w[W], float x[8]) {
    if constexpr (FP8) {
      fp8_values(w[0], x);
      fp8_values(w[1], x + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = act_to_float<ACT>((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
    }
  };
  // the turned piece, fp8 without its scale
  auto turned = [&](const Raw &r, float x[8]) {
    values8(r.own, x);
    if (tby == 0) return;
    float y[8];
    values8(r.other, y);
    const float co[8] = {c[0][0], c[0][1], c[0][2], c[0][3], c[1][0], c[1][1], c[1][2], c[1][3]};
    const float si[8] = {sn[0][0], sn[0][1], sn[0][2], sn[0][3],
                         sn[1][0], sn[1][1], sn[1][2], sn[1][3]};
    if (a.interleaved) turn8<true>(x, y, co, si, false, 1.f);
    else turn8<false>(x, y, co, si, upper, 1.f);
  };

  if (groups == 1) places(0);
  if constexpr (!FP8) {
    Raw next = load(layer0);
    for (int layer = layer0; layer < layer1; ++layer) {
      const Raw r = next;
      if (layer + 1 < layer1) next = load(layer + 1);
      uint8_t *base = a.kv.base + layer * a.layer_bytes;
#pragma unroll
      for (int k = 0; k < KEEP; ++k)
        if (dst[k] >= 0) *reinterpret_cast<u32x4 *>(base + dst[k]) = r.lat[k];
      if (tdst < 0) continue;
      u32x4 w = {r.own[0], r.own[1], r.own[2], r.own[3]};
      if (tby != 0) {
        float x[8];
        turned(r, x);
        w = u32x4{pack_act<ACT>(x[0], x[1]), pack_act<ACT>(x[2], x[3]), pack_act<ACT>(x[4], x[5]),
                  pack_act<ACT>(x[6], x[7])};
      }
      *reinterpret_cast<u32x4 *>(base + tdst) = w;
    }
  } else {
    for (int layer = layer0; layer < layer1; ++layer) {
      uint8_t *base = a.kv.base + layer * a.layer_bytes;
      float amax[2] = {0.f, 0.f};
      Raw r;
      for (int group = 0; group < groups; ++group) {
        if (groups > 1) places(group);
        r = load(layer);
        auto largest = [&](const float *x, int n, float by) {
          float v = 0.f;
#pragma unroll
          for (int i = 0; i < n; ++i) {
            const float y = fabsf(x[i] * by);
            v = fmaxf(v, finite(y) ? y : 0.f);
          }
          return v;
        };
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
          float x[16];
#pragma unroll
          for (int i = 0; i < 4; ++i) fp8_values(r.lat[k][i], x + 4 * i);
          amax[0] = fmaxf(amax[0], largest(x, 16, r.lat_scale[k]));
        }
        float x[8];
        turned(r, x);
        amax[1] = fmaxf(amax[1], largest(x, 8, r.turn_scale));
      }
      float (*to)[2] = most[layer & 1];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        amax[w] = max_wave(amax[w]);
        if ((tid & 63) == 0) to[tid >> 6][w] = amax[w];
      }
      __syncthreads();
      float inv[2];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        float v = to[0][w];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) v = fmaxf(v, to[i][w]);
        const float scale = fp8_scale(v);
        inv[w] = power_inverse(scale);
        if (tid == 0) a.kv.scales[layer * a.layer_scales + (int64_t)m.page * 2 + w] = scale;
      }
      for (int group = 0; group < groups; ++group) {
        if (groups > 1) {
          places(group);
          r = load(layer);
        }
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
          if (dst[k] < 0) continue;
          const float f = factor_of(r.lat_scale[k], inv[0]);
          u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x[4];
            fp8_values(r.lat[k][i], x);
            w[i] = fp8_word(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
          }
          *reinterpret_cast<u32x4 *>(base + dst[k]) = w;
        }
        if (tdst >= 0) {
          const float f = factor_of(r.turn_scale, inv[1]);
          float x[8];
          turned(r, x);
          *reinterpret_cast<u32x2 *>(base + tdst) =
              u32x2{fp8_word(x[0] * f, x[1] * f, x[2] * f, x[3] * f),
                    fp8_word(x[4] * f, x[5] * f, x[6] * f, x[7] * f)};
        }
      }
    }
  }
}

template <int ACT, bool FP8>
hipError_t append(const LatentAppendArgs &a, hipStream_t s) {
  const int64_t blocks = (int64_t)a.b.n_seqs * a.pages_most;
  int64_t grid = blocks;
  if (a.q.data) {
    const int most = heads_of_wave(a.turn / 8);
    const int64_t waves = ((int64_t)a.q_heads + most - 1) / most;
    grid += (a.b.n_rows * waves + kWaves - 1) / kWaves;
  }
  hipLaunchKernelGGL((append_latent<ACT, FP8>), dim3((unsigned)grid), dim3(kThreads), 0, s, a,
                     (uint32_t)blocks);
  return hipGetLastError();
}

template <int ACT, bool FP8>
hipError_t move(const MoveArgs &a, hipStream_t s) {
  const int64_t grid =
      (int64_t)(a.layers + a.layers_wave - 1) / a.layers_wave * a.n_seqs * a.blocks_most;
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
