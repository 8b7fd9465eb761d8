// Attention of many query rows over the paged cache: chunks of a prompt.
//
// The mathematics is the split kernel's; here the matrix products bound it.
// A workgroup of four waves takes 128 rows (query rows times the heads of a
// KV head's group, so a key is loaded once for all of them) and walks the
// tokens in tiles of 64 that its waves share through LDS; a wave keeps 32
// rows.  The products are transposed (S^T = K Q^T, O^T = V^T P^T): a lane
// holds scores of one row only, so the softmax is its own work but for one
// exchange with the lane 32 away, and P goes from the scores' registers into
// the second product as it is.  V^T comes from LDS through transposing reads.
//
// P goes into the second product as one 16-bit value of the type beside it: 8
// bits for bf16 values (the split kernel, whose matrix units idle, takes two),
// 11 for f16 and fp8 ones.  A second product for the rest of P would be half as
// many matrix instructions again in a kernel that they bound.  Against 64 bits
// the chunk below is 0.0023 off (2-norm) where rounding the result alone gives
// 0.0017.  The sums of weights are of the unrounded ones, in 32 bits.
//
// fp8 keys and values become 16-bit values, exactly, on their way into LDS.
// A key's scale multiplies its scores.  A value's scale, relative to the
// largest one among the blocks that the row has seen so far, multiplies its
// weight: both stay 32 bits until the weight is rounded to f16, whose range the
// relative scale and the running maximum hold: down to 2^-29 of both a weight
// keeps 11 bits, below 2^-40 it is gone.
//
// Measured: 2,048 rows of 4 KV heads of 8 over 26,624 16-bit tokens, 0.86
// TFLOP, in 0.92 to 0.95 ms (0.93 PFLOP/s; a large library product reaches
// 1.3), ragged fp8 chunks of 0.22 TFLOP in 0.41 ms.  By counters a SIMD's matrix
// unit is busy for 39% of the former's time and its vector unit for 37%: the
// softmax between the products costs what they do, and two waves a SIMD hide it
// in part.  The ragged chunks' compute units have work for 75% of the time.
#include <hip/hip_runtime.h>

#include "ea_kv_device.hpp"

namespace ea {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kLanes;
constexpr int kTok = kChunkTokens;

// Kinds of instructions for the scheduler, and key reads ahead of a product.
constexpr int kValu = 0x2, kMfma = 0x8, kLdsRead = 0x100, kAhead = 4;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <int ACT, bool FP8, int DT, bool TILES>
__global__ __launch_bounds__(kThreads, DT <= 4 ? 2 : 1) void attend_chunk(AttendArgs a) {
  constexpr int DP = DT * 32;
  constexpr int CH = DP / 8;                  // chunks of 8 elements of a head
  constexpr int PASS = kTok * CH / kThreads;  // chunks a thread stages
  constexpr int STEP = kThreads / CH;         // tokens of a pass
  constexpr int PV = FP8 ? kF16 : ACT;
  constexpr float kShift = PV == kF16 ? 15.f : 0.f;
  constexpr int EB = FP8 ? 1 : 2;
  // pitches: sixteen tokens' 16 bytes of keys, and four tokens' 64 bytes of
  // values, fall on different banks (of 64)
  constexpr int KP = DP * 2 + 16, VP = DP * 2 + 64;
  __shared__ __align__(16) uint8_t k_lds[kTok * KP];
  __shared__ __align__(16) uint8_t v_lds[kTok * VP];
  __shared__ __align__(16) float ks_lds[kTok], vs_lds[kTok];

  const KvLayer &kv = a.kv;
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, gg = lane >> 5;
  const int wave = uniform(tid >> 6);
  const int H = kv.heads, D = kv.head_dim, T = kv.page_tokens, G = a.group;
  const int tiles_most = (a.b.max_rows * G + kChunkRows - 1) / kChunkRows;

  // Tiles of one sequence beside each other read the same keys at about the
  // same time, mostly from an L2 (with sequences beside each other instead,
  // twelve ragged chunks took 508 us for 383); those that see the most tokens
  // start first.
  uint32_t u = blockIdx.x;
  const int h = u % H;
  u /= H;
  const int part = u % a.splits;
  u /= a.splits;
  const int tile = tiles_most - 1 - u % tiles_most;
  const int s = u / tiles_most;
  const Seq sq = sequence(a.b, s);
  if (sq.rows * G <= a.split_rows_most || tile * kChunkRows >= sq.rows * G) return;
  const int pos0 = sq.len - sq.rows;
  const Span span = span_of(a, sq, pos0);
  if (part >= span.parts) return;
  const int32_t *table = a.b.page_table + (int64_t)s * a.b.table_stride;
  const int last_page = sq.len > 0 ? over_page(kv, sq.len - 1) : 0;

  // rows: r of the sequence is query row r / G, head r % G of the group
  const int r = tile * kChunkRows + wave * 32 + c, qi = r / G;
  const bool there = qi < sq.rows;
  const int lim = there ? min(pos0 + qi + 1, sq.len) : 0;
  const int low = there && a.window > 0 ? max(0, pos0 + qi + 1 - a.window) : 0;
  // of the wave's rows: all attend inside [all_low, all_lim), none outside
  // [any_low, any_lim); the workgroup's tokens
  const int q_first = (tile * kChunkRows + wave * 32) / G;
  const int q_last = min((tile * kChunkRows + wave * 32 + 31) / G, sq.rows - 1);
  const int all_lim = min(pos0 + q_first + 1, sq.len);
  const int any_lim = q_first < sq.rows ? min(pos0 + q_last + 1, sq.len) : 0;
  const int all_low = a.window > 0 ? max(0, pos0 + q_last + 1 - a.window) : 0;
  const int any_low = a.window > 0 ? max(0, pos0 + q_first + 1 - a.window) : 0;
  const int wg_first = tile * kChunkRows / G;
  const int wg_last = min((tile * kChunkRows + kChunkRows - 1) / G, sq.rows - 1);
  int t0 = span.begin + part * a.chunk_tokens;
  const int t1 = min(min(span.end, t0 + a.chunk_tokens), pos0 + wg_last + 1);
  const int wg_low = a.window > 0 ? max(0, pos0 + wg_first + 1 - a.window) : 0;
  t0 = max(t0, wg_low & ~(kTok - 1));

  uint32_t qreg[DP / 16][4];
  {
    const uint16_t *qp = a.q.data + (int64_t)(sq.row0 + (there ? qi : 0)) * a.q.row_stride +
                         (int64_t)(h * G + r % G) * a.q.head_stride;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
      const int d = k * 16 + gg * 8;
      u32x4 v = {0, 0, 0, 0};
      if (there && d < D) v = *reinterpret_cast<const u32x4 *>(qp + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) qreg[k][i] = v[i];
    }
  }

  // fp8: O is held in units of v_scale / owed, the change of the unit that O is
  // still to be multiplied by.  A row's own: a unit shared with rows of other
  // blocks would leave small scales beside a large one no bits.
  float m = kNegInf, l = 0.f, v_scale = 0.f, v_inv = 0.f, owed = 1.f;
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;

  const uint32_t token_bytes = H * D * EB, head_at = h * D * EB, piece = (uint32_t)kv.piece;
  const int chunk = tid % CH, first_tok = tid / CH;

  // ---- a tile's keys and values on their way to LDS, and its scales.
  // TILES: 16 tokens share a page, so each of a wave's passes reads one page,
  // as a buffer whose end cuts off what no row attends to (it reads as zero);
  // pages are looked up a tile ahead.  Otherwise lane t looks up token t.
  constexpr uint32_t kPast = 0x80000000u;
  constexpr int TP = kTok / 16;
  uint32_t kr[PASS][FP8 ? 2 : 4], vr[PASS][FP8 ? 2 : 4];
  float k_sc[TILES ? TP : 1] = {}, v_sc[TILES ? TP : 1] = {};
  uint32_t here[TP] = {};  // TILES: pages of the tile to load
  uint64_t gone = 0;       // tokens of the loaded tile whose page is not there
  uint32_t place[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    place[i] = chunk * 8 < D ? ((first_tok + i * 8) & 15) * token_bytes + chunk * 8 * EB : kPast;
  auto look = [&](int base) {
#pragma unroll
    for (int t = 0; t < TP; ++t)
      here[t] = table[(uint32_t)min(over_page(kv, base + t * 16), last_page)];
  };
  auto load = [&](int base) {
    gone = 0;
    if constexpr (TILES) {
      uint32_t page[TP], page_of[TP];
#pragma unroll
      for (int t = 0; t < TP; ++t) {
        page_of[t] = uniform(here[t]);
        const bool ok = page_of[t] < (uint32_t)kv.num_pages;
        page[t] = ok ? page_of[t] : 0;
        if (!ok) gone |= 0xffffull << (16 * t);
        if (FP8) {
          const float *sp =
              kv.scales + ((uint64_t)page[t] * (uint32_t)kv.scale_page + h * kv.scale_head);
          k_sc[t] = sp[0];
          v_sc[t] = ok && base + t * 16 < sq.len && base + t * 16 + 16 > wg_low ? sp[kv.scale_kv]
                                                                               : 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < PASS; ++j) {
        // the pass's 16 tokens, their page and place in it
        const int t = DT == 2 ? (wave >> 1) + 2 * j : j * STEP / 16;
        uint32_t pg = page[0];
#pragma unroll
        for (int i = 1; i < TP; ++i) pg = i == t ? page[i] : pg;
        const int tok = base + t * 16;
        const uint32_t at = uniform((tok - over_page(kv, tok) * T) * token_bytes + head_at);
        const uint32_t held =
            uniform((gone >> (16 * t)) & 1 ? 0 : min(max(sq.len - tok, 0), 16));
        uint8_t *p = kv.base + ((uint64_t)uniform(pg) * piece + at);
        const auto kbuf = __builtin_amdgcn_make_buffer_rsrc(p, 0, held * token_bytes, 0x20000);
        const auto vbuf =
            __builtin_amdgcn_make_buffer_rsrc(p + piece / 2, 0, held * token_bytes, 0x20000);
        const uint32_t off = place[DT == 8 ? j & 1 : 0];
        if constexpr (FP8) {
          const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(kbuf, off, 0, 0);
          const u32x2 y = __builtin_amdgcn_raw_buffer_load_b64(vbuf, off, 0, 0);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            kr[j][i] = x[i];
            vr[j][i] = y[i];
          }
        } else {
          const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(kbuf, off, 0, 0);
          const u32x4 y = __builtin_amdgcn_raw_buffer_load_b128(vbuf, off, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            kr[j][i] = x[i];
            vr[j][i] = y[i];
          }
        }
      }
    } else {
      const int tok = base + lane;
      int p = over_page(kv, tok);
      const int slot0 = tok - p * T;
      const uint32_t page0 = table[(uint32_t)min(p, last_page)];
      const bool there_is = page0 < (uint32_t)kv.num_pages, ok = tok < sq.len && there_is;
      const uint32_t page = ok ? page0 : 0;
      const int slot = ok ? slot0 : -1;
      gone = __ballot(!there_is);
      if (FP8) {
        const float *sp = kv.scales + (uint64_t)page * (uint32_t)kv.scale_page + h * kv.scale_head;
        k_sc[0] = ok ? sp[0] : 0.f;
        v_sc[0] = ok && tok >= wg_low ? sp[kv.scale_kv] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < PASS; ++j) {
        const int t = first_tok + j * STEP;
        const uint32_t pg = __shfl(page, t);
        const int sl = __shfl(slot, t);
        const uint8_t *src = kv.base + ((uint64_t)pg * piece + max(sl, 0) * token_bytes + head_at +
                                        (chunk * 8 < D ? chunk * 8 : 0) * EB);
        const bool in = sl >= 0 && chunk * 8 < D;
        if constexpr (FP8) {
          const u32x2 x = *reinterpret_cast<const u32x2 *>(src);
          const u32x2 y = *reinterpret_cast<const u32x2 *>(src + piece / 2);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            kr[j][i] = in ? x[i] : 0;
            vr[j][i] = in ? y[i] : 0;
          }
        } else {
          const u32x4 x = *reinterpret_cast<const u32x4 *>(src);
          const u32x4 y = *reinterpret_cast<const u32x4 *>(src + piece / 2);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            kr[j][i] = in ? x[i] : 0;
            vr[j][i] = in ? y[i] : 0;
          }
        }
      }
    }
  };

  if (t0 < t1) {
    if (TILES) look(t0);
    load(t0);
    if (TILES) look(t0 + kTok);
  }
  // The rows' units grow to `top`, which is rare.
  auto grow_units = [&](float top) {
    if (!__any(top > v_scale)) return;
    top = fmaxf(top, v_scale);
    owed *= top > 0.f ? v_scale / top : 1.f;
    v_scale = top;
    v_inv = top >= 0x1p-126f ? 1.f / top : 0.f;
  };
  // A weight of zero does not keep out what is not finite: in tiles of which
  // some row does not see all, such values count as zero and are left for the
  // end.
  const int wg_all_lim = min(pos0 + wg_first + 1, sq.len);
  const int wg_all_low = a.window > 0 ? max(0, pos0 + wg_last + 1 - a.window) : 0;
  uint32_t odd = 0;
  for (int base = t0; base < t1; base += kTok) {
    const bool cut = gone || base < wg_all_low || base + kTok > wg_all_lim;
    __syncthreads();  // the last tile has been read
    // TILES: of 16 tokens each; else in LDS, those of values as they are, `most`
    // the largest
    float ks[TP], vs[TP], most = 0.f;
    if (FP8) {
      if (cut) {
#pragma unroll
        for (int t = 0; t < (TILES ? TP : 1); ++t) {
          odd |= !finite(v_sc[t]);
          v_sc[t] = finite(v_sc[t]) ? v_sc[t] : 0.f;
        }
      }
#pragma unroll
      for (int t = 0; t < (TILES ? TP : 1); ++t) {
        ks[t] = k_sc[t] * a.scale_log2;
        vs[t] = v_sc[t];
      }
      if constexpr (TILES) {
        if (cut) {  // of blocks that the row does not see a token of
#pragma unroll
          for (int t = 0; t < TP; ++t)
            vs[t] = base + t * 16 < lim && base + t * 16 + 16 > low ? vs[t] : 0.f;
        }
        float top = 0.f;
#pragma unroll
        for (int t = 0; t < TP; ++t) top = fmaxf(top, fabsf(vs[t]));
        grow_units(top);
#pragma unroll
        for (int t = 0; t < TP; ++t) vs[t] *= v_inv;
      } else {
        most = fabsf(vs[0]);
        for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
        if (wave == 0) {
          ks_lds[lane] = ks[0];
          vs_lds[lane] = vs[0];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < PASS; ++j) {
      const int t = first_tok + j * STEP;
      u32x4 x, y;
      if constexpr (FP8) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          x[2 * i] = fp8_pair<ACT, false>(kr[j][i]);
          x[2 * i + 1] = fp8_pair<ACT, true>(kr[j][i]);
          y[2 * i] = fp8_pair<PV, false>(vr[j][i]);
          y[2 * i + 1] = fp8_pair<PV, true>(vr[j][i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = kr[j][i];
          y[i] = vr[j][i];
        }
      }
      *reinterpret_cast<u32x4 *>(k_lds + t * KP + chunk * 16) = x;
      *reinterpret_cast<u32x4 *>(v_lds + t * VP + chunk * 16) = y;
    }
    if (cut) {  // each thread's own part of the values
      for (int j = 0; j < PASS; ++j) {
        u32x4 *p = reinterpret_cast<u32x4 *>(v_lds + (first_tok + j * STEP) * VP + chunk * 16);
        u32x4 y = *p;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t bad = odd_mask<PV, false>(y[i]);
          odd |= bad;
          y[i] &= ~bad;
        }
        *p = y;
      }
    }
    const uint64_t gone_here = gone;
    __syncthreads();
    if (base + kTok < t1) {
      load(base + kTok);
      if (TILES) look(base + 2 * kTok);
    }
    if (base >= any_lim || base + kTok <= any_low) continue;

    // keys are read from LDS some products ahead of their use
    f32x16 x[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32x4 af =
            *reinterpret_cast<const u32x4 *>(k_lds + (t * 32 + c) * KP + k * 32 + gg * 16);
        x[t] = mfma32<ACT>(af, u32x4{qreg[k][0], qreg[k][1], qreg[k][2], qreg[k][3]}, x[t]);
      }
    __builtin_amdgcn_sched_group_barrier(kLdsRead, kAhead, 0);
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kLdsRead, 1, 0);
    }
    auto scale_of = [&](const float *lds, const float *own, int t, int q) {
      if constexpr (TILES) {
        const float f = own[t * 2 + (q >> 1)];
        return f32x4{f, f, f, f};
      } else {
        return *reinterpret_cast<const f32x4 *>(lds + t * 32 + q * 8 + gg * 4);
      }
    };
    if (FP8) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 f = scale_of(ks_lds, ks, t, q);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[t][q * 4 + i] *= f[i];
        }
    }
    if constexpr (FP8 && !TILES) {
      if (cut) {  // of the tokens that the row sees
        most = 0.f;
#pragma unroll 1  // the scales are read again below: no registers for them
        for (int q = 0; q < 8; ++q) {
          const f32x4 f = *reinterpret_cast<const f32x4 *>(vs_lds + q * 8 + gg * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = base + q * 8 + gg * 4 + i;
            most = fmaxf(most, at >= low && at < lim ? fabsf(f[i]) : 0.f);
          }
        }
        most = max_rows32(most);
      }
      grow_units(most);
    }
    const float unit = FP8 ? 1.f : a.scale_log2;  // of a score, in powers of two
    if (gone_here || base < all_low || base + kTok > all_lim) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = t * 32 + (i >> 2) * 8 + gg * 4 + (i & 3);
          if (base + at < low || base + at >= lim || ((gone_here >> at) & 1))
            x[t][i] = kNegInf;
        }
    }
    float top = m;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x[t][i]);
    top = max_rows32(top);
    const float ref = top == kNegInf ? 0.f : top * unit - kShift;
    if (__any(FP8 ? top != m || owed != 1.f : top != m)) {
      const float f = m == kNegInf ? 0.f : exp2_fast(m * unit - kShift - ref);
      l *= f;
      const float fo = FP8 ? f * owed : f;
      owed = 1.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] *= fo;
      m = top;
    }
    // The weights of 16 tokens are made while the products of the 16 before
    // them run.
    const uint8_t *vp =
        v_lds + (gg * 4 + ((lane & 15) >> 2)) * VP + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int t = k >> 1;
      u32x4 pf;
#pragma unroll
      for (int q2 = 0; q2 < 2; ++q2) {
        const int q = (k & 1) * 2 + q2;
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = exp2_fast(x[t][q * 4 + i] * unit - ref);
          l += p[i];
        }
        if (FP8) {
          f32x4 f = scale_of(vs_lds, vs, t, q);
          if constexpr (!TILES) {
            f *= v_inv;
            // tokens that the row does not see may have any (finite) scale
            if (cut)
#pragma unroll
              for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_fmed3f(f[i], -1.f, 1.f);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] *= f[i];
        }
        pf[q2 * 2] = pack_act<PV>(p[0], p[1]);
        pf[q2 * 2 + 1] = pack_act<PV>(p[2], p[3]);
      }
      // lane of 16: token (lane / 4) and four elements of 16 of a transposing
      // read; it gets one element of four tokens
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint8_t *p = vp + k * 16 * VP + dt * 64;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 8 * VP));
        const u32x2 x0 = __builtin_bit_cast(u32x2, lo), x1 = __builtin_bit_cast(u32x2, hi);
        o[dt] = mfma32<PV>(u32x4{x0[0], x0[1], x1[0], x1[1]}, pf, o[dt]);
      }
    }
    __builtin_amdgcn_sched_group_barrier(kLdsRead, 8, 1);
    __builtin_amdgcn_sched_group_barrier(kValu, FP8 ? 44 : 36, 1);
#pragma unroll
    for (int i = 0; i < 4 * DT; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 1);
      __builtin_amdgcn_sched_group_barrier(kLdsRead, 2, 1);
      __builtin_amdgcn_sched_group_barrier(kValu, (FP8 ? 44 : 36) / DT, 1);
    }
  }

  if (__syncthreads_or(odd != 0)) {
    for (int base = t0; base < t1; base += kTok) {
      const uint32_t own = table[(uint32_t)min(over_page(kv, base + lane), last_page)];
      if (base >= wg_all_low && base + kTok <= wg_all_lim && !__any(own >= (uint32_t)kv.num_pages))
        continue;
      for (int at = base; at < min(base + kTok, t1); ++at) {
        const uint32_t page = __shfl(own, at - base), slot = at - over_page(kv, at) * T;
        if (page >= (uint32_t)kv.num_pages) continue;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int d = dt * 32 + (i >> 2) * 8 + gg * 4 + (i & 3);
            const float v = d < D ? odd_value<ACT, FP8>(kv, page, slot, h, d) : 0.f;
            if (at >= low && at < lim) o[dt][i] += v;
          }
      }
    }
  }

  const float total = add_rows32(l);
  if (!there) return;
  const float unit = FP8 ? 1.f : a.scale_log2;
  const float ref = m == kNegInf ? kNegInf : m * unit - kShift;
  const int64_t row = sq.row0 + qi, head = h * G + r % G;
  // (v_scale 0: only what is not finite has been added)
  const float out_scale = FP8 && v_scale > 0.f ? v_scale * owed : 1.f;
  if (span.parts == 1) {
    const float f = total == 0.f ? 0.f : out_scale / total;
    uint16_t *op = a.out.data + row * a.out.row_stride + head * a.out.head_stride;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int d = dt * 32 + q * 8 + gg * 4;
        if (d >= D) continue;
        *reinterpret_cast<u32x2 *>(op + d) =
            u32x2{pack_act<ACT>(o[dt][q * 4] * f, o[dt][q * 4 + 1] * f),
                  pack_act<ACT>(o[dt][q * 4 + 2] * f, o[dt][q * 4 + 3] * f)};
      }
    if (a.lse && gg == 0)
      a.lse[row * H * G + head] =
          total == 0.f ? kNegInf : (ref + __log2f(total)) * 0.6931471805599453f;
  } else {
    const int64_t at = (row * H * G + head) * a.splits + part;
    float *op = a.part_o + at * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int d = dt * 32 + q * 8 + gg * 4;
        if (d >= D) continue;
        *reinterpret_cast<f32x4 *>(op + d) =
            f32x4{o[dt][q * 4] * out_scale, o[dt][q * 4 + 1] * out_scale,
                  o[dt][q * 4 + 2] * out_scale, o[dt][q * 4 + 3] * out_scale};
      }
    if (gg == 0) {
      a.part_ml[at * 2] = ref;
      a.part_ml[at * 2 + 1] = total;
    }
  }
}

template <int ACT, bool FP8, int DT>
void go(const AttendArgs &a, dim3 grid, dim3 block, hipStream_t s) {
  if (a.kv.page_tokens % 16 == 0)
    hipLaunchKernelGGL((attend_chunk<ACT, FP8, DT, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((attend_chunk<ACT, FP8, DT, false>), grid, block, 0, s, a);
}

template <int ACT, bool FP8>
hipError_t dims(const AttendArgs &a, hipStream_t s) {
  const int64_t tiles = ((int64_t)a.b.max_rows * a.group + kChunkRows - 1) / kChunkRows;
  const dim3 grid((unsigned)(a.b.n_seqs * tiles * a.splits * a.kv.heads)), block(kThreads);
  if (a.kv.head_dim <= 64) go<ACT, FP8, 2>(a, grid, block, s);
  else if (a.kv.head_dim <= 128) go<ACT, FP8, 4>(a, grid, block, s);
  else go<ACT, FP8, 8>(a, grid, block, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_chunk(const AttendArgs &a, int act, int fp8, hipStream_t s) {
  (void)hipGetLastError();
  if (act == kBf16) return fp8 ? dims<kBf16, true>(a, s) : dims<kBf16, false>(a, s);
  return fp8 ? dims<kF16, true>(a, s) : dims<kF16, false>(a, s);
}

}  // namespace ea
