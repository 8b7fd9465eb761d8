// Device helpers of the cache operators' kernels (gfx950).
#pragma once

#include <hip/hip_runtime.h>

#include "ea_kv_ops.hpp"

namespace ea {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kLanes = 64;
constexpr float kNegInf = -__builtin_inff();

__device__ inline uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ inline int32_t uniform(int32_t v) {
  return (int32_t)__builtin_amdgcn_readfirstlane((uint32_t)v);
}
__device__ inline float uniform(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}

__device__ inline int32_t over_page(const KvLayer &kv, int32_t token) {
  return (int32_t)(__umulhi((uint32_t)token << 1, kv.t_mul) >> kv.t_shift);
}

// First row and rows of a sequence, both held to the batch's bounds, and its
// cached tokens.
struct Seq {
  int32_t row0, rows, len;
};
__device__ inline Seq sequence(const BatchRows &b, int32_t s) {
  Seq q;
  if (b.row_start) {
    const int32_t lo = min(max(b.row_start[s], 0), b.n_rows);
    const int32_t hi = min(max(b.row_start[s + 1], lo), b.n_rows);
    q.row0 = lo;
    q.rows = min(hi - lo, b.max_rows);
  } else {
    q.row0 = s;
    q.rows = s < b.n_rows ? 1 : 0;
  }
  q.len = min(max(b.kv_len[s], 0), b.max_kv);
  return q;
}

// The sequence of a row: the last one that starts at or before it.
__device__ inline int32_t sequence_of_row(const BatchRows &b, int32_t row) {
  if (!b.row_start) return row;
  int32_t lo = 0, hi = b.n_seqs - 1;
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) >> 1;
    if (b.row_start[mid] <= row) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The tokens [begin, end) that any row of a sequence attends to, counted
// along the selection where there is one, and the parts the chunk kernel
// splits them into.  Of a selection with more places than the row has blocks
// `end` is what its blocks fill where they come first; listed_of says where
// they end.
struct Span {
  int32_t begin, end, parts;
};
__device__ inline Span span_of(const AttendArgs &a, const Seq &q, int32_t pos) {
  Span s;
  if (a.selected) {  // `pos` is the row's own
    s.begin = 0;
    s.end = pos < 0 ? 0 : min(a.budget, over_page(a.kv, pos) + 1) * a.kv.page_tokens;
  } else {
    const int32_t lowest = q.len - q.rows + 1 - a.window;
    s.begin = a.window > 0 && lowest > 0 ? lowest & ~(kChunkTokens - 1) : 0;
    s.end = q.len;
  }
  s.parts = max(1, (s.end - s.begin + a.chunk_tokens - 1) / a.chunk_tokens);
  return s;
}

// Places of a selection up to its last block at or before `last`.
__device__ inline int32_t listed_of(const int32_t *sel, int32_t budget, int32_t last) {
  constexpr int kAtOnce = 4;  // loads in flight
  const int lane = threadIdx.x & 63;
  for (int32_t top = budget; top > 0; top -= kAtOnce * kLanes) {
    uint32_t e[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int32_t at = top - 1 - i * kLanes - lane;
      e[i] = at < 0 ? ~0u : (uint32_t)sel[at];
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const uint64_t there = __ballot(e[i] <= (uint32_t)last);
      if (there) return top - i * kLanes - __builtin_ctzll(there);
    }
  }
  return 0;
}

// Largest value over the lanes that hold the same column of a 16-column
// (l, l ^ 16, l ^ 32, l ^ 48) or 32-column (l, l ^ 32) tile.
__device__ inline float max_rows32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max_rows16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return max_rows32(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
// A value of the lane CTRL - 0x120 below in a row of 16, around its end.
template <int CTRL>
__device__ inline float row_ror(float v) {
  return __uint_as_float(
      __builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// Largest value over the 16 lanes of a row; over all lanes.
__device__ inline float max_columns(float v) {
  v = fmaxf(v, row_ror<0x128>(v));
  v = fmaxf(v, row_ror<0x124>(v));
  v = fmaxf(v, row_ror<0x122>(v));
  return fmaxf(v, row_ror<0x121>(v));
}
__device__ inline float max_wave(float v) { return max_rows16(max_columns(v)); }
__device__ inline float add_rows32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline float add_rows16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return add_rows32(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Sum over a lane and those below it.
__device__ inline int scan_wave(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return v;
}

// The smallest power of two s >= 2^-126 with top * s >= amax, top = 448 (fp8
// e4m3) or 127 (whole numbers of 8 bits): from the bits, exact.
__device__ inline float power_for(float amax, uint32_t mantissa_top, int32_t log2_top) {
  const uint32_t u = __float_as_uint(amax);
  int32_t e = (int32_t)(u >> 23) - log2_top + ((u & 0x7fffff) > mantissa_top ? 1 : 0);
  // biased exponent of s; a subnormal or zero amax ends at the smallest
  e = min(max(e, 1), 254);
  return __uint_as_float((uint32_t)e << 23);
}
__device__ inline float fp8_scale(float amax) { return power_for(amax, 0x600000, 8); }
__device__ inline float int8_scale(float amax) { return power_for(amax, 0x7e0000, 6); }
// 1 / s of a power of two s in [2^-126, 2^127]; 2^-127 as a subnormal.
__device__ inline float power_inverse(float s) {
  const int32_t e = 254 - (int32_t)(__float_as_uint(s) >> 23);
  return e > 0 ? __uint_as_float((uint32_t)e << 23) : __uint_as_float(0x400000);
}

__device__ inline bool finite(float v) { return (__float_as_uint(v) & 0x7f800000) != 0x7f800000; }

template <int ACT>
struct ActOf;
template <>
struct ActOf<kBf16> {
  typedef __bf16 T;
  typedef bf16x8 V8;
};
template <>
struct ActOf<kF16> {
  typedef _Float16 T;
  typedef f16x8 V8;
};

template <int ACT>
__device__ inline float act_to_float(uint16_t v) {
  return (float)__builtin_bit_cast(typename ActOf<ACT>::T, v);
}
template <int ACT>
__device__ inline uint32_t pack_act(float lo, float hi) {
  typedef typename ActOf<ACT>::T V2 __attribute__((ext_vector_type(2)));
  const V2 v = {(typename ActOf<ACT>::T)lo, (typename ActOf<ACT>::T)hi};  // one instruction
  return __builtin_bit_cast(uint32_t, v);
}

// Two fp8 codes (the low or high half of w) as two 16-bit values, exact.
template <int ACT, bool HIGH>
__device__ inline uint32_t fp8_pair(uint32_t w) {
  if constexpr (ACT == kBf16)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH));
}

// Ones in place of those of a word's two 16-bit values or four fp8 codes that
// are not finite: a one added at the exponent's end (fp8: at the code's end,
// only NaN has all ones) carries into the sign's place.
template <int ACT, bool FP8>
__device__ inline uint32_t odd_mask(uint32_t w) {
  if constexpr (FP8) {
    const uint32_t t = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return (t - (t >> 7)) | t;
  } else {
    const uint32_t t = ((w & 0x7fff7fffu) + (ACT == kBf16 ? 0x00800080u : 0x04000400u)) &
                       0x80008000u;
    return (t - (t >> 15)) | t;
  }
}

// What the value of token `slot` of a page adds to a sum where it, or its
// scale, is not finite; zero where both are.
template <int ACT, bool FP8>
__device__ inline float odd_value(const KvLayer &kv, uint32_t page, uint32_t slot, int h, int d) {
  const uint64_t at = ((uint64_t)slot * kv.heads + h) * kv.head_dim + d;
  const uint8_t *p = kv.base + ((uint64_t)page * (uint32_t)kv.piece + (uint32_t)kv.piece / 2);
  float v;
  if constexpr (FP8) {
    const float scale = kv.scales[(uint64_t)page * (uint32_t)kv.scale_page + h * kv.scale_head +
                                  kv.scale_kv];
    const uint32_t code = p[at] & 0x7f;
    v = finite(scale) ? 0.f : scale;
    if (code == 0x7f || (code == 0 && !finite(scale))) v = __uint_as_float(0x7fc00000u);
    if (p[at] & 0x80) v = -v;
  } else {
    const uint32_t w = reinterpret_cast<const uint16_t *>(p)[at];
    const uint32_t fraction = w & (ACT == kBf16 ? 0x7fu : 0x3ffu);
    v = __uint_as_float((w & 0x8000u) << 16 | 0x7f800000u | (fraction ? 0x400000u : 0));
    if (!odd_mask<ACT, false>(w)) v = 0.f;
  }
  return v;
}

template <int ACT>
__device__ inline f32x4 mfma16(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
  if constexpr (ACT == kBf16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int ACT>
__device__ inline f32x16 mfma32(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
  if constexpr (ACT == kBf16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

__device__ inline float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

}  // namespace ea
