// Attention of few query rows over the paged cache: decode steps, drafted
// tokens, and attention over selected blocks.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(x_j - m),
//   x_j = scale log2(e) (q . k_j),  m the running maximum of x
//
// What bounds it is reading the keys and values once.  A wave takes one KV
// head of one sequence over a part of its tokens, for all the query rows of
// that head (rows times heads of a group are the columns of its matrix
// products), so every cached byte is read by one wave.  A step covers 32
// tokens, and both products are taken transposed:
//
//   S^T = K Q^T   a lane loads the keys of one token of 16 as they lie in
//                 memory; its four results are four tokens of one column
//   O^T = V^T P^T a lane's eight tokens of S^T are the depth of the second
//                 product as they are: any order of the depth serves, so P
//                 stays in its registers.  V^T wants eight tokens of one
//                 element in a lane: the lane loads a run of elements of
//                 each of its eight tokens and transposes in registers by
//                 byte permutes.
//
// So nothing passes through LDS, waves never wait for one another, and the
// next step's keys (values) load while this step's values (keys) are used.
// Matrix units idle for most of the time, which pays for P as a sum of two
// bf16 (16 bits of it) beside bf16 or fp8 values; with f16 values P is one
// f16 (11 bits) held at up to 2^15, so that small weights keep their bits.
#include <hip/hip_runtime.h>

#include "ea_kv_device.hpp"

namespace ea {
namespace {

constexpr int kWaves = 4;

template <int ACT, bool FP8, int VE, int NB, bool TILES>
__global__ __launch_bounds__(kWaves *kLanes) void attend_split(AttendArgs a) {
  constexpr int DP = VE * 16;                 // head dim the registers hold
  constexpr int KL = FP8 ? DP / 64 : DP / 32;  // 16-byte key loads of a tile
  constexpr int KS = DP / 32;                 // products of a tile's scores
  constexpr int VD = FP8 ? VE / 4 : VE / 2;   // words of a token's values
  constexpr int PV = FP8 || ACT == kBf16 ? kBf16 : kF16;
  constexpr int EB = FP8 ? 1 : 2;
  const KvLayer &kv = a.kv;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int H = kv.heads, D = kv.head_dim, T = kv.page_tokens, G = a.group;

  uint32_t u = blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  const int h = u % H;
  u /= H;
  const int part = u % a.splits;
  u /= a.splits;
  const int row_of = a.selected ? (int)(u % a.b.max_rows) : 0;
  const int s = a.selected ? u / a.b.max_rows : u;
  if (s >= a.b.n_seqs) return;
  Seq sq = sequence(a.b, s);
  if (sq.rows * G > a.split_rows_most && !a.selected) return;
  if (row_of >= sq.rows) return;
  const int first_pos = sq.len - sq.rows;  // of the sequence's first row
  int row0 = sq.row0, rows = sq.rows;
  const int32_t *sel = nullptr;
  if (a.selected) {  // a row is alone: its blocks are its own
    row0 += row_of;
    rows = 1;
    sel = a.selected + ((int64_t)row0 * H + h) * a.budget;
  }
  const int pos0 = first_pos + row_of;  // position of this wave's first row
  const Span span = span_of(a, sq, pos0);
  if (part >= span.parts) return;
  const int t0 = span.begin + part * span.each;
  const int t1 = min(span.end, t0 + span.each);
  const int32_t *table = a.b.page_table + (int64_t)s * a.b.table_stride;
  const int last_page = sq.len > 0 ? over_page(kv, sq.len - 1) : 0;

  // columns: row r of the wave is query row r / G, head r % G of the group
  int lim[NB], low[NB];  // a column attends to tokens low <= j < lim
  uint32_t qreg[NB][KS][4];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = nb * 16 + c, qi = r / G;
    const bool there = qi < rows;
    lim[nb] = there ? min(pos0 + qi + 1, sq.len) : 0;
    low[nb] = there && a.window > 0 ? max(0, pos0 + qi + 1 - a.window) : 0;
    const uint16_t *qp = a.q.data + (int64_t)(row0 + (there ? qi : 0)) * a.q.row_stride +
                         (int64_t)(h * G + r % G) * a.q.head_stride;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int d = FP8 ? (k >> 1) * 64 + g * 16 + (k & 1) * 8 : k * 32 + g * 8;
      u32x4 v = {0, 0, 0, 0};
      if (there && d < D) v = *reinterpret_cast<const u32x4 *>(qp + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) qreg[nb][k][i] = v[i];
    }
  }
  // inside [all_low, all_lim) every column attends; outside [any_low,
  // sq.len) none does
  const int all_lim = min(pos0 + 1, sq.len);
  const int all_low = a.window > 0 ? max(0, pos0 + rows - a.window) : 0;
  const int any_low = a.window > 0 ? max(0, pos0 + 1 - a.window) : 0;

  float m[NB], l[NB];
  f32x4 o[NB][VE];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = kNegInf;
    l[nb] = 0.f;
#pragma unroll
    for (int e = 0; e < VE; ++e) o[nb][e] = {0.f, 0.f, 0.f, 0.f};
  }

  // ---- where a step's tokens lie.  TILES: 16 tokens of a tile share a page,
  // and everything about it is uniform.  Otherwise lane c looks up token c of
  // the tile.
  struct Where {
    int32_t page[2], slot[2], tok[2];  // tok: position in the sequence, or
                                       // INT32_MAX where there is none
  };
  auto look = [&](int base) {
    Where w;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int vt = TILES ? base + t * 16 : base + t * 16 + c;
      int p = over_page(kv, vt);
      const int slot = vt - p * T;
      bool ok = vt < t1;
      if (sel) {
        p = ok ? sel[p] : 0;
        ok = ok && p >= 0 && p <= last_page;
      }
      int tok = p * T + slot;
      p = min(max(p, 0), last_page);
      int page = table[p];
      ok = ok && (uint32_t)page < (uint32_t)kv.num_pages;
      w.page[t] = ok ? page : 0;
      w.slot[t] = ok ? slot : 0;
      w.tok[t] = ok ? tok : INT32_MAX;
      if (TILES) {
        w.page[t] = uniform(w.page[t]);
        w.slot[t] = uniform(w.slot[t]);
        w.tok[t] = uniform(w.tok[t]);
      }
    }
    return w;
  };
  const int64_t token_bytes = (int64_t)H * D * EB;
  const int64_t half_piece = kv.piece >> 1;

  u32x4 kb[2][KL];
  auto load_keys = [&](const Where &w) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t *p = kv.base + w.page[t] * kv.piece + w.slot[t] * token_bytes +
                         (int64_t)h * D * EB + (TILES ? c * token_bytes : 0);
#pragma unroll
      for (int j = 0; j < KL; ++j) {
        const int d = FP8 ? j * 64 + g * 16 : j * 32 + g * 8;
        if (DP == D) {
          kb[t][j] = *reinterpret_cast<const u32x4 *>(p + d * EB);
        } else {  // lanes past the head: zeros, nothing read there
          u32x4 v = {0, 0, 0, 0};
          if (FP8 && d + 8 <= D && d + 16 > D) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(p + d);
            v[0] = x[0];
            v[1] = x[1];
          } else if (d < D) {
            v = *reinterpret_cast<const u32x4 *>(p + d * EB);
          }
          kb[t][j] = v;
        }
      }
    }
  };
  uint32_t vb[8][VD];
  auto load_values = [&](const Where &w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = j >> 2, r = g * 4 + (j & 3);
      int page = w.page[t], slot = w.slot[t];
      if (!TILES) {
        page = __shfl(page, r);
        slot = __shfl(slot, r);
      } else {
        slot += r;
      }
      const uint8_t *p = kv.base + page * kv.piece + half_piece + slot * token_bytes +
                         (int64_t)h * D * EB;
      // lanes past the head load its first elements, which go unused
      constexpr int NS = VE > 8 ? 2 : 1, SE = VE / NS, SW = VD / NS;
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const int d = c * VE + n * SE;
        const uint8_t *pd = p + (d < D ? d : 0) * EB;
        if constexpr (SW == 4) {
          const u32x4 x = *reinterpret_cast<const u32x4 *>(pd);
#pragma unroll
          for (int i = 0; i < 4; ++i) vb[j][n * 4 + i] = x[i];
        } else if constexpr (SW == 2) {
          const u32x2 x = *reinterpret_cast<const u32x2 *>(pd);
          vb[j][n * 2] = x[0];
          vb[j][n * 2 + 1] = x[1];
        } else {
          vb[j][n] = *reinterpret_cast<const uint32_t *>(pd);
        }
      }
    }
  };

  if (t0 < t1) {
    Where here = look(t0);
    load_keys(here);
    load_values(here);
    for (int base = t0; base < t1; base += kSplitStep) {
      const bool more = base + kSplitStep < t1;
      const Where next = look(more ? base + kSplitStep : base);
      // positions and scales of this lane's eight tokens
      int tok[8];
      float ks[8], vs[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int t = j >> 2, r = g * 4 + (j & 3);
        if (TILES) tok[j] = here.tok[t] == INT32_MAX ? INT32_MAX : here.tok[t] + r;
        else tok[j] = __shfl(here.tok[t], r);
        ks[j] = a.scale_log2;
        vs[j] = 1.f;
        if (FP8) {
          const int page = TILES ? here.page[t] : __shfl(here.page[t], r);
          const float *sp = kv.scales + (int64_t)page * kv.scale_page + h * kv.scale_head;
          ks[j] *= sp[0];
          vs[j] = sp[kv.scale_kv];
        }
      }
      // scores
      f32x4 x[NB][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) x[nb][t] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          u32x4 af;
          if constexpr (FP8) {
            const uint32_t w0 = kb[t][k >> 1][(k & 1) * 2], w1 = kb[t][k >> 1][(k & 1) * 2 + 1];
            af = u32x4{fp8_pair<ACT, false>(w0), fp8_pair<ACT, true>(w0),
                       fp8_pair<ACT, false>(w1), fp8_pair<ACT, true>(w1)};
          } else {
            af = kb[t][k];
          }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            x[nb][t] = mfma16<ACT>(
                af, u32x4{qreg[nb][k][0], qreg[nb][k][1], qreg[nb][k][2], qreg[nb][k][3]},
                x[nb][t]);
        }
      }
      if (more) load_keys(next);

      bool inside;  // every token counts for every column
      if (TILES) {
        inside = here.tok[0] >= all_low && here.tok[1] >= all_low &&
                 here.tok[0] < all_lim - 15 && here.tok[1] < all_lim - 15;
      } else {
        bool mine = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) mine = mine && tok[j] >= all_low && tok[j] < all_lim;
        inside = __all(mine);
      }
      u32x4 ph[NB], pl[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[nb][j >> 2][j & 3] * ks[j];
        if (!inside) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (tok[j] < low[nb] || tok[j] >= lim[nb]) y[j] = kNegInf;
        }
        float top = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])),
                          fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
        top = fmaxf(max_rows16(top), m[nb]);
        // f16: weights of up to 2^15
        const float ref = top == kNegInf ? 0.f : top - (PV == kF16 ? 15.f : 0.f);
        if (__any(top != m[nb])) {
          const float old = m[nb] == kNegInf ? kNegInf : m[nb] - (PV == kF16 ? 15.f : 0.f);
          const float f = exp2_fast(old - ref);
          l[nb] *= f;
#pragma unroll
          for (int e = 0; e < VE; ++e) o[nb][e] *= f;
          m[nb] = top;
        }
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          p[j] = exp2_fast(y[j] - ref);
          l[nb] += p[j];
          p[j] *= vs[j];
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t hi = pack_act<PV>(p[2 * w], p[2 * w + 1]);
          ph[nb][w] = hi;
          if constexpr (PV == kBf16)
            pl[nb][w] = pack_act<kBf16>(p[2 * w] - __uint_as_float(hi << 16),
                                        p[2 * w + 1] - __uint_as_float(hi & 0xffff0000u));
        }
      }
      // tokens that no column attends to: whatever lies there counts as zero
      if (!inside) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool keep = tok[j] >= any_low && tok[j] < sq.len;
#pragma unroll
          for (int w = 0; w < VD; ++w) vb[j][w] = keep ? vb[j][w] : 0;
        }
      }
#pragma unroll
      for (int w = 0; w < VD; ++w) {
        constexpr int E = FP8 ? 4 : 2;  // elements of a word
        u32x4 af[E];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t v0 = vb[2 * i][w], v1 = vb[2 * i + 1][w];
          if constexpr (FP8) {
            const uint32_t p01 = __builtin_amdgcn_perm(v1, v0, 0x05010400);
            const uint32_t p23 = __builtin_amdgcn_perm(v1, v0, 0x07030602);
            af[0][i] = fp8_pair<PV, false>(p01);
            af[1][i] = fp8_pair<PV, true>(p01);
            af[2][i] = fp8_pair<PV, false>(p23);
            af[3][i] = fp8_pair<PV, true>(p23);
          } else {
            af[0][i] = __builtin_amdgcn_perm(v1, v0, 0x05040100);
            af[1][i] = __builtin_amdgcn_perm(v1, v0, 0x07060302);
          }
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            o[nb][w * E + e] = mfma16<PV>(af[e], ph[nb], o[nb][w * E + e]);
            if constexpr (PV == kBf16)
              o[nb][w * E + e] = mfma16<PV>(af[e], pl[nb], o[nb][w * E + e]);
          }
      }
      if (more) load_values(next);
      here = next;
    }
  }

#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const float total = add_rows16(l[nb]);
    const int r = nb * 16 + c, qi = r / G;
    if (qi >= rows) continue;
    const int64_t row = row0 + qi, head = h * G + r % G;
    const float ref = m[nb] == kNegInf ? kNegInf : m[nb] - (PV == kF16 ? 15.f : 0.f);
    if (span.parts == 1) {
      const float f = total == 0.f ? 0.f : 1.f / total;
      uint16_t *op = a.out.data + row * a.out.row_stride + head * a.out.head_stride;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int e = 0; e < VE; e += 4) {
          const int d = (g * 4 + i) * VE + e;
          if (d >= D) continue;
          const u32x2 v = {
              pack_act<ACT>(o[nb][e][i] * f, o[nb][e + 1][i] * f),
              pack_act<ACT>(o[nb][e + 2][i] * f, o[nb][e + 3][i] * f)};
          *reinterpret_cast<u32x2 *>(op + d) = v;
        }
      }
      if (a.lse && g == 0)
        a.lse[row * H * G + head] =
            total == 0.f ? kNegInf : (ref + __log2f(total)) * 0.6931471805599453f;
    } else {
      const int64_t at = (row * H * G + head) * a.splits + part;
      float *op = a.part_o + at * D;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int e = 0; e < VE; e += 4) {
          const int d = (g * 4 + i) * VE + e;
          if (d >= D) continue;
          *reinterpret_cast<f32x4 *>(op + d) =
              f32x4{o[nb][e][i], o[nb][e + 1][i], o[nb][e + 2][i], o[nb][e + 3][i]};
        }
      }
      if (g == 0) {
        a.part_ml[at * 2] = ref;
        a.part_ml[at * 2 + 1] = total;
      }
    }
  }
}

// Join of a row's parts: o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i.
// One wave a row and head; parts beside each other in the workspace.
template <int ACT>
__global__ __launch_bounds__(kWaves *kLanes) void attend_join(AttendArgs a) {
  const int HQ = a.kv.heads * a.group, D = a.kv.head_dim;
  const int lane = threadIdx.x & 63;
  const int64_t u = (int64_t)blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  if (u >= (int64_t)a.b.n_rows * HQ) return;
  const int row = u / HQ, head = u % HQ;
  const int s = sequence_of_row(a.b, row);
  const Seq sq = sequence(a.b, s);
  if (row < sq.row0 || row >= sq.row0 + sq.rows) return;
  const Span span = span_of(a, sq, sq.len - sq.rows + row - sq.row0);
  if (span.parts <= 1) return;
  const float *ml = a.part_ml + u * a.splits * 2;
  const float *po = a.part_o + u * a.splits * D;
  float top = kNegInf;
  for (int i = lane; i < span.parts; i += kLanes) top = fmaxf(top, ml[2 * i]);
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float ref = top == kNegInf ? 0.f : top;
  float total = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const int d0 = lane * 4;
  for (int i = 0; i < span.parts; ++i) {
    const float f = exp2_fast(ml[2 * i] - ref);
    total += f * ml[2 * i + 1];
    if (d0 < D) acc += f * *reinterpret_cast<const f32x4 *>(po + (int64_t)i * D + d0);
  }
  const float f = total == 0.f ? 0.f : 1.f / total;
  if (d0 < D) {
    const u32x2 v = {pack_act<ACT>(acc[0] * f, acc[1] * f),
                     pack_act<ACT>(acc[2] * f, acc[3] * f)};
    *reinterpret_cast<u32x2 *>(a.out.data + (int64_t)row * a.out.row_stride +
                               (int64_t)head * a.out.head_stride + d0) = v;
  }
  if (a.lse && lane == 0)
    a.lse[u] = total == 0.f ? kNegInf : (ref + __log2f(total)) * 0.6931471805599453f;
}

template <int ACT, bool FP8, int VE, int NB>
hipError_t go(const AttendArgs &a, hipStream_t s) {
  const int64_t units = (int64_t)a.b.n_seqs * (a.selected ? a.b.max_rows : 1) * a.splits *
                        a.kv.heads;
  const dim3 grid((unsigned)((units + kWaves - 1) / kWaves)), block(kWaves * kLanes);
  if (a.kv.page_tokens % 16 == 0)
    hipLaunchKernelGGL((attend_split<ACT, FP8, VE, NB, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((attend_split<ACT, FP8, VE, NB, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <int ACT, bool FP8, int VE>
hipError_t columns(const AttendArgs &a, hipStream_t s) {
  const int most = (a.selected ? 1 : a.b.max_rows) * a.group;
  const int cols = most < a.split_rows_most ? most : a.split_rows_most;
  if (cols <= 16) return go<ACT, FP8, VE, 1>(a, s);
  if constexpr (VE <= 8) {
    if (cols <= 32) return go<ACT, FP8, VE, 2>(a, s);
    if (cols <= 64) return go<ACT, FP8, VE, 4>(a, s);
  }
  return hipErrorInvalidValue;
}

template <int ACT, bool FP8>
hipError_t dims(const AttendArgs &a, hipStream_t s) {
  if (a.kv.head_dim <= 64) return columns<ACT, FP8, 4>(a, s);
  if (a.kv.head_dim <= 128) return columns<ACT, FP8, 8>(a, s);
  return columns<ACT, FP8, 16>(a, s);
}

}  // namespace

hipError_t launch_attend_split(const AttendArgs &a, int act, int fp8, hipStream_t s) {
  (void)hipGetLastError();
  if (act == kBf16) return fp8 ? dims<kBf16, true>(a, s) : dims<kBf16, false>(a, s);
  return fp8 ? dims<kF16, true>(a, s) : dims<kF16, false>(a, s);
}

hipError_t launch_attend_join(const AttendArgs &a, int act, hipStream_t s) {
  (void)hipGetLastError();
  const int64_t units = (int64_t)a.b.n_rows * a.kv.heads * a.group;
  const dim3 grid((unsigned)((units + kWaves - 1) / kWaves)), block(kWaves * kLanes);
  if (act == kBf16) hipLaunchKernelGGL(attend_join<kBf16>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(attend_join<kF16>, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace ea
