// What the kernels that write blocks of a cache share: a lane's place in a
// token's head, stored values, fp8 codes, a block's bounds.
#pragma once

#include <hip/hip_runtime.h>

#include "ea_kv_device.hpp"

namespace ea {

// Lanes side by side on one token's head, two pieces of 8 elements each.
constexpr int lanes_of(int head_dim) { return head_dim <= 64 ? 4 : head_dim <= 128 ? 8 : 16; }

template <int ACT>
__device__ inline void read8(const uint16_t *p, float x[8]) {
  const u32x4 v = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = act_to_float<ACT>((uint16_t)(v[i >> 1] >> (16 * (i & 1))));
}

// What a lane has of every head: elements d[0] ..+7 and d[1] ..+7, and whether
// the head has them.  Rotation pairs i with i + dim / 2: where that is whole
// pieces, a lane has both halves of its pairs.
struct Place {
  int d[2];
  bool in[2];
  bool paired;  // its two pieces turn together
};
__device__ inline Place place_of(int lp, int D, bool turn, int dim, bool interleaved) {
  Place p;
  const int half = dim >> 1;
  const bool halves = turn && !interleaved && (half & 7) == 0;
  p.paired = halves && lp * 8 < half;
  if (p.paired) {
    p.d[0] = lp * 8;
    p.d[1] = lp * 8 + half;
  } else {  // neighbours: of what does not turn, or of the whole head
    p.d[0] = halves ? dim + (lp * 8 - half) * 2 : lp * 16;
    p.d[1] = p.d[0] + 8;
  }
  p.in[0] = p.d[0] < D;
  p.in[1] = p.d[1] < D;
  return p;
}

// Cosines and sines of a lane's pairs at a position.
struct Angles {
  f32x4 c[2], s[2];
};
__device__ inline Angles angles_of(const float *rope, int pos, int dim, const Place &p) {
  Angles a = {};
  if (p.paired) {
    const float *cs = rope + (int64_t)pos * dim + p.d[0], *sn = cs + (dim >> 1);
    a.c[0] = *reinterpret_cast<const f32x4 *>(cs);
    a.c[1] = *reinterpret_cast<const f32x4 *>(cs + 4);
    a.s[0] = *reinterpret_cast<const f32x4 *>(sn);
    a.s[1] = *reinterpret_cast<const f32x4 *>(sn + 4);
  }
  return a;
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

// What takes codes of scale `by` to those of a new block, 1 / inv its scale: exact,
// as inv is a power of two.  Beside codes that are all zeros it may pass 32 bits
// (one that is not gives the new block a scale that keeps it below 2^19), and zeros
// times infinity are NaN: it stays finite where `by` is.
__device__ inline float factor_of(float by, float inv) {
  constexpr float kMost = 0x1.fffffep127f;
  const float f = by * inv;
  return finite(by) ? fmaxf(fminf(f, kMost), -kMost) : f;
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

// Of two values, the larger over the lane and the one 32 (16) away: the first's
// in the lower of the two, the second's in the upper.
__device__ inline float max_halves32(float a, float b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max_halves16(float a, float b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Largest values of 16 elements over the lanes with the same place in groups of
// LP: those of elements 4 * (lane / 16 in the order 0, 1, 2, 3) + 0 .. 3.
template <int LP>
__device__ inline void max_tokens16(const float v[16], float out[4]) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = max_halves32(v[i], v[8 + i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y = max_halves16(x[i], x[4 + i]);
    if constexpr (LP <= 8) y = fmaxf(y, row_ror<0x128>(y));
    if constexpr (LP <= 4) y = fmaxf(y, row_ror<0x124>(y));
    out[i] = y;
  }
}

// Bounds of a block's keys as whole numbers: lowest rounded down, highest
// rounded up, in units of a power of two that holds them within 127.  LP lanes
// hold a token's head; every (64 / LP)-th token is a lane's, its lowest and
// highest elements in lo and hi.  Values that are not finite do not set the
// unit; an infinity is the largest whole number.  The reduction over tokens
// leaves a lane four elements, whose bounds it makes and writes.
template <int LP>
__device__ inline void write_bounds(const KvLayer &kv, int page, int h, int lane, const Place &p,
                                    float lo[16], float hi[16]) {
  const int D = kv.head_dim;
  const int q = lane >> 4, d = (q >> 1 ? p.d[1] : p.d[0]) + (q & 1) * 4;
  const bool in = q >> 1 ? p.in[1] : p.in[0];
  float l[4], u[4], amax = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) lo[i] = -lo[i];
  max_tokens16<LP>(lo, l);
  max_tokens16<LP>(hi, u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (in && finite(l[i])) amax = fmaxf(amax, fabsf(l[i]));
    if (in && finite(u[i])) amax = fmaxf(amax, fabsf(u[i]));
  }
  const float s = int8_scale(max_wave(amax)), inv = power_inverse(s);
  if (in && (lane & 15) < LP) {
    uint32_t wl = 0, wh = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int a = (int)fmaxf(fminf(floorf(-l[i] * inv), 127.f), -127.f);
      const int b = (int)fmaxf(fminf(ceilf(u[i] * inv), 127.f), -127.f);
      wl |= (uint32_t)(uint8_t)a << (8 * i);
      wh |= (uint32_t)(uint8_t)b << (8 * i);
    }
    int8_t *to = kv.bounds + ((int64_t)page * 2 * kv.heads + h) * D + d;
    *reinterpret_cast<uint32_t *>(to) = wl;
    *reinterpret_cast<uint32_t *>(to + (int64_t)kv.heads * D) = wh;
  }
  if (lane == 0) kv.bound_scales[(int64_t)page * kv.heads + h] = s;
}

// A sequence's moved tokens from `first` on, `most` at most: n tokens from list
// place `at` on, their first new position; n 0: none.  Of a block, its page too.
struct MovedBlock {
  int32_t page, n, at;
  int64_t pos;
  const int32_t *table;  // of the old pages
};
__device__ inline MovedBlock moved_run(const MoveArgs &a, int s, int first, int most) {
  const int lo = min(max(a.token_start[s], 0), a.n_tokens);
  const int hi = min(max(a.token_start[s + 1], lo), a.n_tokens);
  MovedBlock m = {-1, min(min(hi - lo, a.max_tokens) - first, most), lo + first,
                  (int64_t)(a.dst_first ? a.dst_first[s] : 0) + first,
                  a.src_table + (int64_t)s * a.src_stride};
  return m;
}
__device__ inline MovedBlock moved_block(const MoveArgs &a, int s, int j) {
  MovedBlock m = moved_run(a, s, j * a.kv.page_tokens, a.kv.page_tokens);
  if (m.n <= 0) return m;
  const int page = a.dst_table[(int64_t)s * a.dst_stride + j];
  if ((uint32_t)page >= (uint32_t)a.kv.num_pages) m.n = 0;
  m.page = page;
  return m;
}

// Where token i of the block was, and how far it moves.  page -1: nowhere.
struct MovedToken {
  int32_t page, slot, by;
};
__device__ inline MovedToken moved_token(const MoveArgs &a, const MovedBlock &m, int i) {
  MovedToken t = {-1, 0, 0};
  const int old = a.tokens[m.at + i];
  if ((uint32_t)old >= (uint32_t)a.max_kv) return t;
  const int e = over_page(a.kv, old);
  const int64_t by = m.pos + i - old;
  const int page = m.table[e];
  if ((uint32_t)page >= (uint32_t)a.kv.num_pages) return t;
  if (a.rope && (by >= a.rope_len || by <= -(int64_t)a.rope_len)) return t;
  t.page = page;
  t.slot = old - e * a.kv.page_tokens;
  t.by = a.rope ? (int32_t)by : 0;
  return t;
}

}  // namespace ea
