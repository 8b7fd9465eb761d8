// Attention of few query rows over the paged cache: decode steps, drafted
// tokens, and attention over selected blocks.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(x_j - m),
//   x_j = scale log2(e) (q . k_j),  m the running maximum of x
//
// What bounds it is reading the keys and values once.  A workgroup takes one
// KV head of one sequence over a part of its tokens, for all the query rows of
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
// So nothing passes through LDS on the way, and the next step's keys (values)
// load while this step's values (keys) are used.  The waves of a
// workgroup take a run of the part's tokens each and become one result in
// LDS; a long context's parts are joined by the workgroup that ends last.
// Matrix units idle for most of the time, which pays for P as a sum of two
// bf16 (16 bits of it) beside bf16 or fp8 values; with f16 values P is one
// f16 (11 bits) held at up to 2^15, so that small weights keep their bits.
//
// Measured: 64 sequences of 8,192-65,536 fp8 tokens, one KV head of 8, 623 MB
// in 114 us (5.5 TB/s; reading random pages alone reaches 6.0); one sequence
// of 4 KV heads and 65,536 16-bit tokens, 134 MB, in 33 us, of which some 10
// are the launch, the first loads' latency and the join.
#include <hip/hip_runtime.h>

#include "ea_kv_device.hpp"

namespace ea {
namespace {

// Parts that a workgroup of the same launch joins pass between the chip's
// L2 caches, one for each XCD.  They are written and read as relaxed atomics
// of agent scope, which go past those caches, and a workgroup counts itself
// once its writes are done (s_waitcnt vmcnt(0) in every wave, then the
// barrier).  Agent-scope fences say the same but write back and drop the
// whole L2 each time: with them 64 contexts of 8,192-65,536 fp8 tokens took
// 372 us, 4 heads of 65,536 16-bit tokens 130 us.
__device__ inline void put_part(float *p, float x, float y) {
  const uint64_t v = (uint64_t)__float_as_uint(x) | ((uint64_t)__float_as_uint(y) << 32);
  __hip_atomic_store(reinterpret_cast<uint64_t *>(p), v, __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline f32x2 get_part(const float *p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  return f32x2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}

// A workgroup's part of a unit that others have parts of: for each of its
// heads `cols` rows of D sums, then the rows' references and totals.
__device__ inline float *part_at(const AttendArgs &a, int wg, int cols) {
  return a.split_parts + (int64_t)wg * a.heads_wg * cols * (a.kv.head_dim + 2);
}

// Counts a workgroup whose part is written; true, in all its threads, for
// the last of `of`.  The counter goes back to zero for the next call.
__device__ inline bool last_of(int32_t *counter, int of, int32_t *shared) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const int32_t n = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT);
    if (n == of - 1)
      __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *shared = n;
  }
  __syncthreads();
  return *shared == of - 1;
}

// Join of `parts` (kJoin at most) parts of a unit, those of workgroups w0,
// w0 + stride, ..:
//   o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i,  m = max_i m_i.
// Lanes take four elements of a row.  `last`: the result is the row's output,
// else it takes the first part's place.
constexpr int kJoin = 8;
template <int ACT, int DP, int W>
__device__ inline void join_parts(const AttendArgs &a, int w0, int stride, int parts, int cols,
                                  int row0, int rows, int h0, bool last) {
  constexpr int LP = DP / 4, NG = W * kLanes / LP;
  const int D = a.kv.head_dim, G = a.group, R = rows * G, lp = threadIdx.x % LP;
  const int d0 = lp * 4, dr = d0 < D ? d0 : 0, sums = a.heads_wg * cols * D;
  for (int i = threadIdx.x / LP; i < a.heads_wg * R; i += NG) {
    const int hw = i / R, of = i - hw * R, r = hw * cols + of;  // row `of` of the head
    f32x2 ml[kJoin], x[kJoin], y[kJoin];
#pragma unroll
    for (int k = 0; k < kJoin; ++k) {
      const float *p = part_at(a, w0 + min(k, parts - 1) * stride, cols);
      ml[k] = get_part(p + sums + 2 * r);
      x[k] = get_part(p + r * D + dr);
      y[k] = get_part(p + r * D + dr + 2);
    }
    float ref = kNegInf, total = 0.f;
#pragma unroll
    for (int k = 0; k < kJoin; ++k) ref = fmaxf(ref, ml[k][0]);
    const float zero = ref == kNegInf ? 0.f : ref;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kJoin; ++k) {
      if (k < parts) {
        const float f = exp2_fast(ml[k][0] - zero);
        total += f * ml[k][1];
        acc += f * f32x4{x[k][0], x[k][1], y[k][0], y[k][1]};
      }
    }
    if (!last) {
      float *p = part_at(a, w0, cols);
      if (d0 < D) {
        put_part(p + r * D + d0, acc[0], acc[1]);
        put_part(p + r * D + d0 + 2, acc[2], acc[3]);
      }
      if (lp == 0) put_part(p + sums + 2 * r, ref, total);
      continue;
    }
    const float f = total == 0.f ? 0.f : 1.f / total;
    const int64_t row = row0 + of / G, head = (h0 + hw) * G + of % G;
    if (d0 < D)
      *reinterpret_cast<u32x2 *>(a.out.data + row * a.out.row_stride +
                                 head * a.out.head_stride + d0) =
          u32x2{pack_act<ACT>(acc[0] * f, acc[1] * f), pack_act<ACT>(acc[2] * f, acc[3] * f)};
    if (a.lse && lp == 0)
      a.lse[row * a.kv.heads * G + head] =
          total == 0.f ? kNegInf : (ref + __log2f(total)) * 0.6931471805599453f;
  }
}

// The work of a call in steps of 32 tokens for each run of a workgroup: a
// sequence has `units` units (heads_wg KV heads; with selections, a row and
// its KV head) of `steps` steps each.  Every wave of every workgroup finds the
// same totals from the sequences' lengths, which only the device knows.
struct SeqWork {
  Seq q;
  int32_t units, steps;
};
template <int W>
__device__ inline SeqWork work_of(const AttendArgs &a, int s) {
  SeqWork w = {{0, 0, 0}, 0, 0};
  if (s >= a.b.n_seqs) return w;
  w.q = sequence(a.b, s);
  if (w.q.rows == 0 || (!a.selected && w.q.rows * a.group > a.split_rows_most)) return w;
  const Span sp = span_of(a, w.q, w.q.len - 1);  // the last row's selection is the longest
  w.units = a.kv.heads / a.heads_wg * (a.selected ? w.q.rows : 1);
  const int step = W / a.heads_wg * kSplitStep;
  w.steps = max(1, (sp.end - sp.begin + step - 1) / step);
  return w;
}

template <int ACT, bool FP8, int VE, int NB, bool TILES>
__global__ __launch_bounds__(split_waves(VE * 16, NB * 16) * kLanes,
                             split_waves(VE * 16, NB * 16) / 4 *
                                 split_resident(VE * 16, NB * 16)) void
attend_split(AttendArgs a) {
  constexpr int W = split_waves(VE * 16, NB * 16);
  constexpr int DP = VE * 16;                 // head dim the registers hold
  constexpr int KL = FP8 ? DP / 64 : DP / 32;  // 16-byte key loads of a tile
  constexpr int KS = DP / 32;                 // products of a tile's scores
  constexpr int VD = FP8 ? VE / 4 : VE / 2;   // words of a token's values
  constexpr int PV = FP8 || ACT == kBf16 ? kBf16 : kF16;
  constexpr float kShift = PV == kF16 ? 15.f : 0.f;
  constexpr int EB = FP8 ? 1 : 2;
  constexpr int NS = TILES ? 2 : 8;           // scales of a step a lane holds
  __shared__ float wave_ml[W][NB * 16][2];
  __shared__ float wave_o[W][VE * 4][kLanes];
  __shared__ int32_t arrived;

  const KvLayer &kv = a.kv;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = uniform((int)threadIdx.x >> 6);
  const int H = kv.heads, D = kv.head_dim, T = kv.page_tokens, G = a.group;

  // ---- this workgroup's unit and part.  A unit comes in as many equal parts
  // as keep each within `each` steps: the share of a workgroup where all have
  // the same, or as much more as makes the parts fit the workgroups
  const int HW = a.heads_wg, HG = H / HW;
  SeqWork sw = work_of<W>(a, lane);  // of sequence `lane`
  int all = sw.units * sw.steps;
  for (int s0 = kLanes; s0 < a.b.n_seqs; s0 += kLanes) {
    const SeqWork w = work_of<W>(a, s0 + lane);
    all += w.units * w.steps;
  }
  all = __builtin_amdgcn_readlane(scan_wave(all), kLanes - 1);
  int each = a.least_steps ? max(parts_of_steps(all, a.split_wgs), a.least_steps) : INT32_MAX;
  for (int i = 0; a.least_steps && a.b.n_seqs <= kLanes; ++i) {
    const int n = __builtin_amdgcn_readlane(
        scan_wave(sw.units * parts_of_steps(sw.steps, each)), kLanes - 1);
    if (n <= a.split_wgs || i == 3) break;
    each = each + max(1, (int)((float)each * (n - a.split_wgs) / a.split_wgs));
  }
  int s = -1, unit = blockIdx.x, parts = 1;  // unit: within the sequence, times parts
  Seq sq = {0, 0, 0};
  int steps = 0;
  for (int s0 = 0; s0 < a.b.n_seqs; s0 += kLanes) {
    if (s0) sw = work_of<W>(a, s0 + lane);
    const int in = parts_of_steps(sw.steps, each);
    const int upto = scan_wave(sw.units * in);
    const uint64_t found = __ballot(unit < upto);
    if (found) {
      const int l = __builtin_ctzll(found);
      s = s0 + l;
      parts = __builtin_amdgcn_readlane(in, l);
      unit -= __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(sw.units, l) * parts;
      steps = __builtin_amdgcn_readlane(sw.steps, l);
      sq.row0 = __builtin_amdgcn_readlane(sw.q.row0, l);
      sq.rows = __builtin_amdgcn_readlane(sw.q.rows, l);
      sq.len = __builtin_amdgcn_readlane(sw.q.len, l);
      break;
    }
    unit -= __builtin_amdgcn_readlane(upto, kLanes - 1);
  }
  if (s < 0) return;
  const int part = unit % parts, h0 = unit / parts % HG * HW, row_of = unit / parts / HG;
  // the wave's head, and its run of the part's tokens
  const int hw = wave % HW, h = h0 + hw, runs = W / HW, my_run = wave / HW;
  const int first_pos = sq.len - sq.rows;  // of the sequence's first row
  int row0 = sq.row0, rows = sq.rows;
  const int32_t *sel = nullptr;
  if (a.selected) {  // a row is alone: its blocks are its own
    row0 += row_of;
    rows = 1;
    sel = a.selected + ((int64_t)row0 * H + h) * a.budget;
  }
  const int pos0 = first_pos + row_of;  // position of the first row
  Span span = span_of(a, sq, pos0);
  const int step = runs * kSplitStep;
  if (sel && pos0 >= 0 && span.end < a.budget * T) {
    // skipped places may come before blocks.  Looked for only where there are
    // more places than blocks: 64 contexts of 300 tokens with 128 places 10.6
    // -> 11.4 us; walking every place instead 23.9
    span.end = listed_of(sel, a.budget, over_page(kv, pos0)) * T;
    steps = (span.end + step - 1) / step;
  }
  // this part's steps and tokens, and the wave's of them
  const int share = steps / parts, more_for = steps % parts;
  const int from = part * share + min(part, more_for);
  const int to = from + share + (part < more_for ? 1 : 0);
  const int run = (to - from) * kSplitStep;
  const int p0 = span.begin + from * step, p1 = min(span.end, span.begin + to * step);
  const int t0 = p0 + my_run * run, t1 = min(p1, t0 + run);
  const int32_t *table = a.b.page_table + (int64_t)s * a.b.table_stride;
  const int last_page = sq.len > 0 ? over_page(kv, sq.len - 1) : 0;

  // columns: row r is query row r / G, head r % G of the group
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

  // ---- where a step's tokens lie, in three stages of a load each, so that
  // each is asked for a step before it is needed: the token's entry in the page
  // table (a selection is a list of entries), its page, the page's scales.
  // TILES: 16 tokens of a tile share a page, and everything about it is
  // uniform.  Otherwise lane c looks up token c of the tile.
  struct Entries {
    int32_t e[2], slot[2], vt[2];
  };
  struct Paged {
    uint32_t page[2], slot[2];
    int32_t tok[2];  // position in the sequence, INT32_MAX where there is none
  };
  const int32_t last_entry = over_page(kv, max(p1 - 1, 0));
  auto entries = [&](int base) {
    Entries r;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      r.vt[t] = base + t * 16 + (TILES ? 0 : c);
      const int32_t e = over_page(kv, r.vt[t]);
      r.slot[t] = r.vt[t] - e * T;
      r.e[t] = sel ? sel[(uint32_t)min(e, last_entry)] : min(e, last_entry);
    }
    return r;
  };
  auto pages = [&](const Entries &r) {
    Paged w;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bool ok = r.vt[t] < t1 && (uint32_t)r.e[t] <= (uint32_t)last_page;
      w.slot[t] = r.slot[t];
      w.tok[t] = ok ? r.e[t] * T + r.slot[t] : INT32_MAX;
      w.page[t] = table[ok ? (uint32_t)r.e[t] : 0u];
    }
    return w;
  };
  auto checked = [&](Paged w) {  // a page outside the cache holds no tokens
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bool ok = w.page[t] < (uint32_t)kv.num_pages;
      w.page[t] = ok ? w.page[t] : 0;
      w.tok[t] = ok ? w.tok[t] : INT32_MAX;
    }
    return w;
  };
  struct Scales {
    float k[NS], v[NS];
  };
  const float *head_scales = kv.scales + h * kv.scale_head;
  auto scales_of = [&](const Paged &w) {
    Scales x;
#pragma unroll
    for (int j = 0; j < NS; ++j) {
      x.k[j] = x.v[j] = 1.f;
      if (FP8) {
        const uint32_t page = TILES ? w.page[j] : __shfl(w.page[j >> 2], g * 4 + (j & 3));
        const float *sp = head_scales + (uint64_t)page * (uint32_t)kv.scale_page;
        x.k[j] = sp[0];
        x.v[j] = sp[kv.scale_kv];
      }
    }
    return x;
  };
  // places inside a page are 32 bits
  const uint32_t token_bytes = H * D * EB, head_at = h * D * EB, piece = (uint32_t)kv.piece;

  // ---- loads.  TILES: a page is a buffer, a lane's place in it the same in
  // every tile; elements past the head lie past the buffer's end and read as
  // zero, and so does a tile that holds no tokens, whose buffer is empty.
  constexpr uint32_t kPast = 0x80000000u;
  constexpr int kNt = 2;  // the load's nt bit: not to be kept in the caches
  auto buffer_of = [&](const Paged &w, int t) {
    const uint32_t at = w.slot[t] * token_bytes + head_at;
    return __builtin_amdgcn_make_buffer_rsrc(kv.base + ((uint64_t)w.page[t] * piece + at), 0,
                                             w.tok[t] == INT32_MAX ? 0 : (int)(piece - at),
                                             0x20000);
  };
  uint32_t key_off[KL], value_off[4][VE > 8 ? 2 : 1];
  if (TILES) {
#pragma unroll
    for (int j = 0; j < KL; ++j) {
      const int d = FP8 ? j * 64 + g * 16 : j * 32 + g * 8;
      key_off[j] = d < D ? (uint32_t)(c * token_bytes) + d * EB : kPast;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int n = 0; n < (VE > 8 ? 2 : 1); ++n) {
        const int d = c * VE + n * 8;
        value_off[i][n] = d < D ? (uint32_t)((g * 4 + i) * token_bytes) + d * EB : kPast;
      }
  }
  u32x4 kb[2][KL];
  auto load_keys = [&](const Paged &w) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (TILES) {
        const auto buf = buffer_of(w, t);
#pragma unroll
        for (int j = 0; j < KL; ++j)
          kb[t][j] = __builtin_amdgcn_raw_buffer_load_b128(
              buf, key_off[j], 0, 0);
      } else {
        const uint8_t *p =
            kv.base + ((uint64_t)w.page[t] * piece + w.slot[t] * token_bytes + head_at);
#pragma unroll
        for (int j = 0; j < KL; ++j) {
          const int d = FP8 ? j * 64 + g * 16 : j * 32 + g * 8;
          u32x4 v = {0, 0, 0, 0};
          if (FP8 && d + 8 == D) {
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
  auto load_values = [&](const Paged &w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = j >> 2, r = g * 4 + (j & 3);
      constexpr int NP = VE > 8 ? 2 : 1, SW = VD / NP;  // pieces, words of a piece
      const auto buf = buffer_of(w, t);
      const uint8_t *p = nullptr;
      if (!TILES)
        p = kv.base + ((uint64_t)__shfl(w.page[t], r) * piece + piece / 2 +
                       __shfl(w.slot[t], r) * token_bytes + head_at);
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        // lanes past the head: its first elements, which go unused
        const int d = c * VE + n * 8;
        const uint8_t *pd = p + (d < D ? d : 0) * EB;
        if constexpr (SW == 4) {
          u32x4 x;
          if (TILES) x = __builtin_amdgcn_raw_buffer_load_b128(buf, value_off[j & 3][n],
                                                               (int)(piece / 2), kNt);
          else x = *reinterpret_cast<const u32x4 *>(pd);
#pragma unroll
          for (int i = 0; i < 4; ++i) vb[j][n * 4 + i] = x[i];
        } else if constexpr (SW == 2) {
          u32x2 x;
          if (TILES) x = __builtin_amdgcn_raw_buffer_load_b64(buf, value_off[j & 3][n],
                                                              (int)(piece / 2), kNt);
          else x = *reinterpret_cast<const u32x2 *>(pd);
          vb[j][n * 2] = x[0];
          vb[j][n * 2 + 1] = x[1];
        } else {
          if (TILES) vb[j][n] = __builtin_amdgcn_raw_buffer_load_b32(buf, value_off[j & 3][n],
                                                                     (int)(piece / 2), kNt);
          else vb[j][n] = *reinterpret_cast<const uint32_t *>(pd);
        }
      }
    }
  };

  // whether every token of a step counts for every column
  auto inside_of = [&](const Paged &w) {
    if (TILES)
      return w.tok[0] >= all_low && w.tok[1] >= all_low && w.tok[0] < all_lim - 15 &&
             w.tok[1] < all_lim - 15;
    return (bool)__all(w.tok[0] >= all_low && w.tok[1] >= all_low && w.tok[0] < all_lim &&
                       w.tok[1] < all_lim);
  };
  uint32_t odd = 0;  // where some do not: whether a value there is not finite

  if (t0 < t1) {
    Paged here = checked(pages(entries(t0)));
    Paged ahead = pages(entries(t0 + kSplitStep));
    Entries far = entries(t0 + 2 * kSplitStep);
    Scales sc = scales_of(here);
    // keys before values, as in the loop: the wait for the keys leaves the
    // values in flight
    load_keys(here);
    __builtin_amdgcn_sched_barrier(0);
    load_values(here);
    __builtin_amdgcn_sched_barrier(0);
    for (int base = t0; base < t1; base += kSplitStep) {
      const Paged next = checked(ahead);
      const Scales sc_next = scales_of(next);
      ahead = pages(far);
      far = entries(base + 3 * kSplitStep);
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
      load_keys(next);

      // position of this lane's token j
      auto tok = [&](int j) {
        const int t = j >> 2, r = g * 4 + (j & 3);
        if (!TILES) return __shfl(here.tok[t], r);
        return here.tok[t] == INT32_MAX ? INT32_MAX : here.tok[t] + r;
      };
      const bool inside = inside_of(here);
      if (FP8 && !inside) {
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          odd |= !finite(sc.v[j]);
          sc.v[j] = finite(sc.v[j]) ? sc.v[j] : 0.f;
        }
      }
      u32x4 ph[NB], pl[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          y[j] = x[nb][j >> 2][j & 3] *
                 (FP8 ? sc.k[TILES ? j >> 2 : j] * a.scale_log2 : a.scale_log2);
        if (!inside) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int at = tok(j);
            if (at < low[nb] || at >= lim[nb]) y[j] = kNegInf;
          }
        }
        float top = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])),
                          fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
        top = fmaxf(max_rows16(top), m[nb]);
        // f16: weights of up to 2^15
        const float ref = top == kNegInf ? 0.f : top - kShift;
        if (__any(top != m[nb])) {
          const float f = m[nb] == kNegInf ? 0.f : exp2_fast(m[nb] - kShift - ref);
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
          if (FP8) p[j] *= sc.v[TILES ? j >> 2 : j];
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
      // A weight of zero does not keep out what is not finite: tokens that no
      // column attends to count as zero, and of the others such values are
      // left for the end.
      if (!inside) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int at = tok(j);
          const bool keep = at >= any_low && at < sq.len;
#pragma unroll
          for (int w = 0; w < VD; ++w) {
            const uint32_t v = keep ? vb[j][w] : 0, bad = odd_mask<ACT, FP8>(v);
            odd |= bad;
            vb[j][w] = v & ~bad;
          }
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
      load_values(next);
      here = next;
      sc = sc_next;
    }
  }

  // ---- values that are not finite, where not every column attends to them
  if (__any(odd != 0)) {
    for (int base = t0; base < t1; base += kSplitStep) {
      const Paged w = checked(pages(entries(base)));
      if (inside_of(w)) continue;
      for (int j = 0; j < kSplitStep; ++j) {
        const int t = j >> 4, r = j & 15;
        const uint32_t page_of = t ? w.page[1] : w.page[0], slot_of = t ? w.slot[1] : w.slot[0];
        int at = t ? w.tok[1] : w.tok[0];
        const uint32_t page = TILES ? page_of : __shfl(page_of, r);
        const uint32_t slot = TILES ? slot_of + r : __shfl(slot_of, r);
        if (!TILES) at = __shfl(at, r);
        if (at == INT32_MAX) continue;
        if (TILES) at += r;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const int d = (g * 4 + i) * VE + e;
            const float v = d < D ? odd_value<ACT, FP8>(kv, page, slot, h, d) : 0.f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              if (at >= low[nb] && at < lim[nb]) o[nb][e][i] += v;
          }
      }
    }
  }

  float *mine_at = part_at(a, blockIdx.x, NB * 16);
  // ---- the runs of a head become one result
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const float total = add_rows16(l[nb]);
    if (g == 0) {
      wave_ml[wave][nb * 16 + c][0] = m[nb] == kNegInf ? kNegInf : m[nb] - kShift;
      wave_ml[wave][nb * 16 + c][1] = total;
    }
  }
  __syncthreads();
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    // reference and total of head hw0 + `of`
    auto statistics = [&](int of, float &ref, float &total) {
      ref = kNegInf;
      total = 0.f;
      for (int w = of; w < W; w += HW) ref = fmaxf(ref, wave_ml[w][nb * 16 + c][0]);
      const float zero = ref == kNegInf ? 0.f : ref;
      for (int w = of; w < W; w += HW)
        total += exp2_fast(wave_ml[w][nb * 16 + c][0] - zero) * wave_ml[w][nb * 16 + c][1];
    };
    float ref, total;
    statistics(hw, ref, total);
    const float f = exp2_fast(wave_ml[wave][nb * 16 + c][0] - (ref == kNegInf ? 0.f : ref));
    if (nb) __syncthreads();  // the last columns have been read
#pragma unroll
    for (int e = 0; e < VE; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) wave_o[wave][i * VE + e][lane] = o[nb][e][i] * f;
    __syncthreads();
    const int r = nb * 16 + c, qi = r / G;
    // a wave sums and writes a quarter of a head's elements, (g * 4 + i) * VE
    // ..+VE-1 of lane (c, g)
    for (int t = wave; t < HW * 4; t += W) {
      const int of = t % HW, i = t / HW, d0 = (g * 4 + i) * VE;
      if (HW > 1) statistics(of, ref, total);
      if (qi < rows) {
        float v[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = 0.f;
        for (int w = of; w < W; w += HW)
#pragma unroll
          for (int e = 0; e < VE; ++e) v[e] += wave_o[w][i * VE + e][lane];
        const int64_t row = row0 + qi, head = (h0 + of) * G + r % G;
        if (parts == 1) {
          const float norm = total == 0.f ? 0.f : 1.f / total;
          uint16_t *op = a.out.data + row * a.out.row_stride + head * a.out.head_stride;
#pragma unroll
          for (int e = 0; e < VE; e += 4)
            if (d0 + e < D)
              *reinterpret_cast<u32x2 *>(op + d0 + e) =
                  u32x2{pack_act<ACT>(v[e] * norm, v[e + 1] * norm),
                        pack_act<ACT>(v[e + 2] * norm, v[e + 3] * norm)};
          if (a.lse && g == 0 && i == 0)
            a.lse[row * H * G + head] =
                total == 0.f ? kNegInf : (ref + __log2f(total)) * 0.6931471805599453f;
        } else {
          float *op = mine_at + (of * NB * 16 + r) * D;
#pragma unroll
          for (int e = 0; e < VE; e += 4)
            if (d0 + e < D) {
              put_part(op + d0 + e, v[e], v[e + 1]);
              put_part(op + d0 + e + 2, v[e + 2], v[e + 3]);
            }
          if (g == 0 && i == 0)
            put_part(mine_at + HW * NB * 16 * D + 2 * (of * NB * 16 + r), ref, total);
        }
      }
    }
  }
  if (parts == 1) return;
  // ---- eight parts are joined by the workgroup of them that ends last, then
  // eight of those, and so on: counting on one address is serial (64 parts on
  // one counter took 10 us, twice as many twice that)
  const int w0 = blockIdx.x - part;
  for (int stride = 1, level = 0;; stride *= kJoin, ++level) {
    const int at = part / (stride * kJoin) * (stride * kJoin);  // first of the eight
    const int of = min((parts - at + stride - 1) / stride, kJoin);
    const bool last = parts <= stride * kJoin;
    if (of > 1) {
      // the counter `level` after that of the first of the eight
      if (!last_of(a.arrivals + w0 + at + level, of, &arrived)) return;
      join_parts<ACT, DP, W>(a, w0 + at, stride, of, NB * 16, row0, rows, h0, last);
    }
    if (last) return;
  }
}

constexpr int kJoinWaves = 4;

// Join of the chunk kernel's parts: one wave a row and head, a lane four
// elements.  It reads the parts once, a launch of its own after the products
// (18 us of 407 for six ragged fp8 chunks).
template <int ACT>
__global__ __launch_bounds__(kJoinWaves *kLanes) void attend_join(AttendArgs a) {
  const int HQ = a.kv.heads * a.group, D = a.kv.head_dim;
  const int lane = threadIdx.x & 63;
  const int64_t u = (int64_t)blockIdx.x * kJoinWaves + uniform(threadIdx.x >> 6);
  if (u >= (int64_t)a.b.n_rows * HQ) return;
  const int row = u / HQ, head = u % HQ;
  const int s = sequence_of_row(a.b, row);
  const Seq sq = sequence(a.b, s);
  if (row < sq.row0 || row >= sq.row0 + sq.rows) return;
  if (sq.rows * a.group <= a.split_rows_most) return;  // not the chunk kernel's
  const int parts = span_of(a, sq, sq.len - 1).parts;
  if (parts <= 1) return;
  const float *ml = a.part_ml + u * a.splits * 2;
  const float *po = a.part_o + u * a.splits * D;
  float top = kNegInf;
  for (int i = lane; i < parts; i += kLanes) top = fmaxf(top, ml[2 * i]);
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float ref = top == kNegInf ? 0.f : top;
  float total = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const int d0 = lane * 4, dr = d0 < D ? d0 : 0;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) {
    const float f = exp2_fast(ml[2 * i] - ref);
    total += f * ml[2 * i + 1];
    acc += f * *reinterpret_cast<const f32x4 *>(po + (int64_t)i * D + dr);
  }
  const float f = total == 0.f ? 0.f : 1.f / total;
  if (d0 < D)
    *reinterpret_cast<u32x2 *>(a.out.data + (int64_t)row * a.out.row_stride +
                               (int64_t)head * a.out.head_stride + d0) =
        u32x2{pack_act<ACT>(acc[0] * f, acc[1] * f), pack_act<ACT>(acc[2] * f, acc[3] * f)};
  if (a.lse && lane == 0)
    a.lse[u] = total == 0.f ? kNegInf : (ref + __log2f(total)) * 0.6931471805599453f;
}

template <int ACT, bool FP8, int VE, int NB>
hipError_t go(const AttendArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.split_grid), block(split_waves(VE * 16, NB * 16) * kLanes);
  // tiles of 16 tokens inside a page, 16-byte pieces inside a head
  if (a.kv.page_tokens % 16 == 0 && (!FP8 || a.kv.head_dim % 16 == 0))
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
  const dim3 grid((unsigned)((units + kJoinWaves - 1) / kJoinWaves)), block(kJoinWaves * kLanes);
  if (act == kBf16) hipLaunchKernelGGL(attend_join<kBf16>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(attend_join<kF16>, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace ea
