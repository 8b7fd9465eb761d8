// Attention over a cache of latents: of absorbed queries, whose keys are a
// token's whole row (latent and turned part) and whose values are its latent.
//
//   o = sum_j p_j c_j / sum_j p_j,  p_j = 2^(x_j - m),
//   x_j = scale log2(e) (q_c . c_j + q_r . r_j),  m a reference near the maximum
//
// All query heads share a token's row, so the rows of a matrix product are
// query rows times heads, and a cached byte feeds both products: 2 (2 C + R) H
// operations for (C + R) e bytes, 1.9 a byte for each head (C 512, R 64, 16 bits),
// so that a row of 16 heads is bound by memory, one of 128 (242 a byte) by both
// alike, and more rows by the products.
//
// Both products are turned around, S^T = K Q^T and O^T = V^T P^T: a column is a
// row's head, a lane has one column's statistics, and the weights come out of the
// first product as the second one's operand takes them, without a way through LDS.
// A workgroup is one wave for each SIMD, which has its 512 registers: 32 columns'
// queries (144) and sums (256, in the accumulation registers), of 512 elements.  So
// a tile of rows is read from LDS once for each 32 columns.  Rows go to LDS as they
// are stored, by loads that write no register; keys are read in rows, values with
// transposing reads, of places swapped so that no two lanes meet in a bank
// (counted: no conflicts).
//
// The reference m of a row moves only when a score is more than 2^8 above it, so
// the sums are rarely rescaled; statistics and sums have 32 bits.  Weights are
// rounded to 11 bits beside f16 and fp8 values (up to 2^15: 7 of shift, 8 of
// slack).  Beside bf16 ones they are the sum of two bf16, 16 bits, where sequences
// have at most 64 columns: the two waves of four that would have none take the
// others' columns with the second bf16, and the sums become one at the end (TWO;
// 24 sequences of 2-4 rows of 16 heads 101 us with one bf16, 108 with two; the
// second in the same wave, half of the products anew: 119).  With more columns they are
// rounded to 8 bits, as the products bound the kernel there: half a step, 2^-8, of
// each, of random signs in a sum, as the result's own rounding is.  An fp8 value's
// scale goes into its weight before that.
//
// Measured (C 512, R 64, pages of 16 tokens in random order), the join included:
// 64 sequences of 8,192-65,536 tokens, a row of 16 heads, fp8: 305 us (4.6 TB/s; its
// loads alone 266); 2,048 rows of 16 heads over 26,624 tokens, bf16: 1.60-1.68 ms
// (1.09-1.14 PFLOP/s; without its loads 1.29 ms); 65,536 tokens, a row of 128 heads,
// bf16: 65 us, 42-46 of them before the join; 24 sequences of 2-4 rows, bf16: 97 us.
#include <hip/hip_runtime.h>

#include "ea_kv_device.hpp"

namespace ea {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kLanes;
constexpr int kTurn = 64;      // elements of a row's turned part that the registers hold
constexpr int kRing = 147456;  // most bytes of tokens in LDS

__device__ const u32x4 kZeros = {0, 0, 0, 0};

// 16 bytes a lane from base + off (from p) to LDS, lane by lane from `at` on, if
// `there` is not zero; of the lanes in `lanes`.  The load writes no register, and
// the compiler does not know of it: whoever reads the bytes waits for it (vmcnt).
// All lanes are active where these stand.  (Changing them takes as long as the
// products before it, so that only what needs it does.)
__device__ inline void to_lds(uint32_t at, const uint8_t *base, uint32_t off, uint32_t there) {
  asm volatile("s_cmp_eq_u32 %3, 0\n\ts_cbranch_scc1 .Lpast%=\n\ts_mov_b32 m0, %0\n\t"
               "s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n.Lpast%=:"
               :
               : "s"(uniform(at)), "v"(off), "s"(base), "s"(uniform(there))
               : "memory", "scc");
}
__device__ inline void to_lds_some(uint32_t at, const uint8_t *p, uint32_t there,
                                   uint64_t lanes) {
  asm volatile("s_cmp_eq_u32 %2, 0\n\ts_cbranch_scc1 .Lpast%=\n\ts_mov_b32 m0, %0\n\t"
               "s_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %1, off\n\t"
               "s_mov_b64 exec, -1\n.Lpast%=:"
               :
               : "s"(uniform(at)), "v"(p), "s"(uniform(there)), "s"(lanes)
               : "memory", "scc");
}
// A value that has arrived.  The compiler waits for its own loads where their
// values are used: in the steps' loop it would wait for the rows on their way too.
template <typename V>
__device__ inline void here(V &v) {
  asm volatile("" : "+v"(v));
}
template <int N>
__device__ inline void wait_loads() {
  static_assert(N >= 0 && N < 64, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ inline void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

// A product into vector registers: the sums of O take the accumulation
// registers, and the compiler puts results of its own matrix instructions there.
// It does not know what these are, so they bring the waits that the hardware asks
// for: two cycles after a vector instruction may have written an operand, sixteen
// before one reads the results (settled()).  ZERO: not added to anything.
template <int ACT, bool ZERO>
__device__ inline void multiply32(f32x16 &x, const u32x4 &v, const u32x4 &w) {
  if constexpr (ACT == kBf16 && ZERO)
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(x) : "v"(v), "v"(w));
  else if constexpr (ACT == kBf16)
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(x) : "v"(v), "v"(w));
  else if constexpr (ZERO)
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(x) : "v"(v), "v"(w));
  else
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(x) : "v"(v), "v"(w));
}
__device__ inline void settled(f32x16 &x) { asm volatile("s_nop 15" : "+v"(x)); }

// Sums times f, in their accumulation registers.  Rare, so it waits for any
// matrix instruction before and behind it.
template <int DT>
__device__ inline void rescale(f32x16 (&o)[DT], float f) {
  asm volatile("s_nop 15\n\ts_nop 7" : : : "memory");
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      float t0 = o[dt][i], t1 = o[dt][i + 1], t2 = o[dt][i + 2], t3 = o[dt][i + 3], tmp;
      asm volatile("v_accvgpr_read_b32 %4, %0\n\tv_mul_f32 %4, %4, %5\n\t"
                   "v_accvgpr_write_b32 %0, %4\n\t"
                   "v_accvgpr_read_b32 %4, %1\n\tv_mul_f32 %4, %4, %5\n\t"
                   "v_accvgpr_write_b32 %1, %4\n\t"
                   "v_accvgpr_read_b32 %4, %2\n\tv_mul_f32 %4, %4, %5\n\t"
                   "v_accvgpr_write_b32 %2, %4\n\t"
                   "v_accvgpr_read_b32 %4, %3\n\tv_mul_f32 %4, %4, %5\n\t"
                   "v_accvgpr_write_b32 %3, %4"
                   : "+a"(t0), "+a"(t1), "+a"(t2), "+a"(t3), "=&v"(tmp)
                   : "v"(f));
      o[dt][i] = t0;
      o[dt][i + 1] = t1;
      o[dt][i + 2] = t2;
      o[dt][i + 3] = t3;
    }
  asm volatile("s_nop 7" : : : "memory");
}

// Four sums of a tile with something added, likewise.
__device__ inline void add4(f32x16 &o, int i4, const float (&add)[4]) {
  float t0 = o[i4 * 4], t1 = o[i4 * 4 + 1], t2 = o[i4 * 4 + 2], t3 = o[i4 * 4 + 3], tmp;
  asm volatile("v_accvgpr_read_b32 %4, %0\n\tv_add_f32 %4, %4, %5\n\t"
               "v_accvgpr_write_b32 %0, %4\n\t"
               "v_accvgpr_read_b32 %4, %1\n\tv_add_f32 %4, %4, %6\n\t"
               "v_accvgpr_write_b32 %1, %4\n\t"
               "v_accvgpr_read_b32 %4, %2\n\tv_add_f32 %4, %4, %7\n\t"
               "v_accvgpr_write_b32 %2, %4\n\t"
               "v_accvgpr_read_b32 %4, %3\n\tv_add_f32 %4, %4, %8\n\t"
               "v_accvgpr_write_b32 %3, %4"
               : "+a"(t0), "+a"(t1), "+a"(t2), "+a"(t3), "=&v"(tmp)
               : "v"(add[0]), "v"(add[1]), "v"(add[2]), "v"(add[3]));
  o[i4 * 4] = t0;
  o[i4 * 4 + 1] = t1;
  o[i4 * 4 + 2] = t2;
  o[i4 * 4 + 3] = t3;
}

__device__ inline float of_lane(float v, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}

struct SeqTiles {
  Seq q;
  int32_t units, steps;
};

// A sequence's units (tiles of its rows times heads) and steps of each.
template <int QW, int STEP>
__device__ inline SeqTiles tiles_of(const LatentAttendArgs &a, int s) {
  SeqTiles w = {{0, 0, 0}, 0, 0};
  if (s >= a.b.n_seqs) return w;
  w.q = sequence(a.b, s);
  if (w.q.rows == 0) return w;
  w.units = (int32_t)(((int64_t)w.q.rows * a.q_heads + QW * 32 - 1) / (QW * 32));
  w.steps = max(1, (w.q.len + STEP - 1) / STEP);
  return w;
}

// Pages and rows: runs of 16 tokens inside pages and whole rows that the
// registers hold (kPlain), other rows (kRows), other pages (kPages).  A launch's
// smallest row is padded to 256 or 512 elements and 64 with zeros, which cost
// products but no bytes.
enum Mode { kPlain, kRows, kPages };

template <int ACT, bool FP8, int CT, int QW, Mode MODE, bool TWO>
__global__ __launch_bounds__(kThreads, 1) void attend_latent(LatentAttendArgs a) {
  constexpr int KG = kWaves / QW;        // groups of waves that share tokens
  constexpr int STEP = KG * 32;          // tokens of a step, 32 a group
  static_assert(STEP == latent_step(QW), "the host counts the same steps");
  constexpr bool WHOLE = MODE != kPages;
  constexpr int EB = FP8 ? 1 : 2;
  constexpr int RC = CT * EB, RR = kTurn * EB;  // bytes of a token's parts in LDS
  constexpr int TILE = 32 * (RC + RR), STAGE = KG * TILE;
  constexpr int NST = kRing / STAGE < 4 ? kRing / STAGE : 4;  // steps in LDS
  constexpr bool PIPE = NST > 2;         // the next tile's scores beside this one's weights
  constexpr int KC = RC / 32, KR = RR / 32, KN = KC + KR;  // 16-byte reads of a tile's keys
  constexpr int KS = (CT + kTurn) / 16;  // products of a tile's scores
  constexpr int DT = CT / 32, VB = 8 / EB;      // tiles of O; of them in 16 pieces
  constexpr int AHEAD = 4, VAHEAD = 3;   // reads of keys, values ahead of their use
  constexpr int PV = FP8 ? kF16 : ACT;
  constexpr float kShift = PV == kF16 ? 7.f : 0.f, kSlack = 8.f;
  constexpr int LPR = RC / 16, RPI = kLanes / LPR, NI = 8 / RPI;  // loads of 8 tokens' latents
  constexpr int EIGHTS = 4 / QW;         // eights of tokens that a wave loads in a step
  constexpr int LOADS = EIGHTS * (NI + 1);
  static_assert(NST >= 2 && LOADS * (NST > 2 ? NST - 2 : 1) < 64, "shape of the ring");
  constexpr int CR = CT / 2;             // elements of a round of the waves' join
  constexpr int JOIN = KG > 1 ? kWaves * 32 * CR * 4 : 0;
  constexpr int BYTES = NST * STAGE > JOIN ? NST * STAGE : JOIN;
  __shared__ __align__(1024) uint8_t ring[BYTES];
  __shared__ float wave_ml[kWaves][32][2];

  const KvLayer &kv = a.kv;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4, c = lane & 31, h = lane >> 5;
  const int wave = uniform((int)threadIdx.x >> 6);
  const int qg = wave % QW, kg = wave / QW;
  const int HQ = a.q_heads, T = kv.page_tokens, C = a.latent, R = a.turn;
  const uint32_t row_bytes = (C + R) * EB;

  // ---- this workgroup's unit and part, as many equal parts of a unit as keep
  // each within `each` steps: the share of a workgroup where all have the
  // same, or as much more as makes the parts fit the workgroups
  SeqTiles sw = tiles_of<QW, STEP>(a, lane);
  int all = sw.units * sw.steps;
  for (int s0 = kLanes; s0 < a.b.n_seqs; s0 += kLanes) {
    const SeqTiles w = tiles_of<QW, STEP>(a, s0 + lane);
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
  int s = -1, unit = blockIdx.x, parts = 1;
  Seq sq = {0, 0, 0};
  int units = 0;
  for (int s0 = 0; s0 < a.b.n_seqs; s0 += kLanes) {
    if (s0) sw = tiles_of<QW, STEP>(a, s0 + lane);
    const int in = parts_of_steps(sw.steps, each);
    const int upto = scan_wave(sw.units * in);
    const uint64_t found = __ballot(unit < upto);
    if (found) {
      const int l = __builtin_ctzll(found);
      s = s0 + l;
      parts = __builtin_amdgcn_readlane(in, l);
      units = __builtin_amdgcn_readlane(sw.units, l);
      unit -= __builtin_amdgcn_readlane(upto, l) - units * parts;
      sq.row0 = __builtin_amdgcn_readlane(sw.q.row0, l);
      sq.rows = __builtin_amdgcn_readlane(sw.q.rows, l);
      sq.len = __builtin_amdgcn_readlane(sw.q.len, l);
      break;
    }
    unit -= __builtin_amdgcn_readlane(upto, kLanes - 1);
  }
  if (s < 0) return;
  // tiles that see the most tokens start first
  const int part = unit % parts, r0 = (units - 1 - unit / parts) * (QW * 32);
  const int rows_all = sq.rows * HQ, pos0 = sq.len - sq.rows;
  const int q_first = r0 / HQ, q_last = (min(r0 + QW * 32, rows_all) - 1) / HQ;
  // rows see at least all_lim tokens, at most `end`
  const int all_lim = max(min(pos0 + q_first + 1, sq.len), 0);
  const int end = max(min(pos0 + q_last + 1, sq.len), 0);
  const int steps = (end + STEP - 1) / STEP, share = steps / parts, more_for = steps % parts;
  const int from = part * share + min(part, more_for);
  const int part_steps = share + (part < more_for ? 1 : 0), p0 = from * STEP;
  // the wave's: where it has its tokens to itself it stops at the last one
  const int n_steps = uniform(
      QW > 1 ? part_steps : min(part_steps, max(0, (end - p0 - kg * 32 + STEP - 1) / STEP)));
  const int32_t *table = a.b.page_table + (int64_t)s * a.b.table_stride;
  const int last_entry = over_page(kv, max(end - 1, 0));

  // ---- queries, the second operand of S = K Q^T: column c
  // (TWO: of waves 0 and 1; the others have the same columns, and of their weights
  // what the first bf16 leaves)
  const int cg = TWO ? qg & 1 : qg, my = r0 + cg * 32 + c, my_q = my / HQ;
  const bool second = TWO && qg > 1;
  const bool mine = my < rows_all;
  u32x4 qreg[KS];
  {
    const uint16_t *qp = a.q.data + (int64_t)(sq.row0 + (mine ? my_q : 0)) * a.q.row_stride +
                         (int64_t)(mine ? my - my_q * HQ : 0) * a.q.head_stride;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int d = FP8 ? (k >> 1) * 32 + h * 16 + (k & 1) * 8 : k * 16 + h * 8;
      const bool in = mine && (d < CT ? d < C : d - CT < R);
      const uint16_t *p = qp + (d < CT ? d : C + d - CT);
      qreg[k] = *reinterpret_cast<const u32x4 *>(
          in ? p : reinterpret_cast<const uint16_t *>(&kZeros));
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) here(qreg[k]);
  }
  const int lim = mine ? min(pos0 + my_q + 1, sq.len) : INT32_MAX;

  // the n-th tile of O that sixteen tokens add to: those whose values lie whole
  // 256 bytes apart one after another
  auto tile_of_sum = [](int n) { return n % (DT / VB) * VB + n / (DT / VB); };

  // ---- where tokens lie.  A group's run n is 16 tokens from run_at(n) on, two of
  // them a step.  Pages of whole runs: lane l looks up run n0 + l; else token
  // l % 16 of run n0 + l / 16.
  constexpr int BATCH = WHOLE ? kLanes : kLanes / 16;
  auto run_at = [&](int n) { return p0 + ((n >> 1) * KG + kg) * 32 + (n & 1) * 16; };
  auto look = [&](int n0, uint32_t &page, int &slot) {
    const int tok = WHOLE ? run_at(n0 + lane) : run_at(n0 + (lane >> 4)) + c16;
    const int e = over_page(kv, min(tok, max(end - 1, 0)));
    const uint32_t pg = table[min(e, last_entry)];
    slot = max(min(tok, end - 1), 0) - e * T;
    page = tok < end && pg < (uint32_t)kv.num_pages ? pg : ~0u;
    here(page);
    here(slot);
  };

  // ---- loads.  A token's 16-byte pieces lie in LDS in another order for each
  // of sixteen tokens, so that what is read at once falls on different banks (of
  // 64): one piece of tokens 0-3, 12-15, 20-27 or of the others (keys; measured to
  // be the lanes of 16-byte reads that go together), four neighbouring ones of four
  // tokens, or two of 0-3 and 8-11 (values, 16 bits and fp8).
  auto swap_of = [](int row) {
    return FP8 ? (row & 3) << 1 | (row & 8) | ((row >> 2) & 1) : (row & 3) << 2 | ((row >> 2) & 3);
  };
  auto turn_swap_of = [](int row) { return FP8 ? (row >> 2) & 3 : (row >> 1) & 7; };
  const uint32_t ring_at = uniform((uint32_t)(uintptr_t)(lds_u8 *)ring);
  constexpr int TL = RR / 16;  // lanes of a token's turned part
  // (the swap of a sum of rows whose bits differ is the swaps' together)
  // a load takes the turned parts of eight tokens, in fp8 of all of a run
  const int lat_row = lane / LPR, turn_row = lane / TL;
  const uint32_t lat_piece = ((lane % LPR) ^ swap_of(lat_row)) << 4,
                 turn_piece = ((lane % TL) ^ turn_swap_of(turn_row)) << 4;
  uint32_t load_page = ~0u;
  int load_slot = 0, load_n0 = -(1 << 20);
  // Eight tokens that the wave is to load: `from` the first's row (a zero where
  // there is none), rows up to `last`, which takes the place of those behind it;
  // nobody attends to these.
  struct Eight {
    const uint8_t *from;
    uint32_t to;  // the tile
    int at, last, at_n;
    uint32_t rows, there;  // all ones, or zero
  };
  auto eight_of = [&](int step, int e) {
    const int eight = qg + QW * e, n = step * 2 + (eight >> 1);
    if (n - load_n0 >= BATCH) {
      load_n0 = n - n % BATCH;
      look(load_n0, load_page, load_slot);
    }
    Eight x;
    x.at = eight * 8;
    x.to = ring_at + (step % NST) * STAGE + kg * TILE;
    x.at_n = n - load_n0;
    x.there = step < n_steps;
    if constexpr (WHOLE) {
      const uint32_t page = __builtin_amdgcn_readlane(load_page, x.at_n);
      const uint32_t slot = __builtin_amdgcn_readlane(load_slot, x.at_n);
      x.rows = page == ~0u ? 0 : ~0u;
      x.last = min(max(end - run_at(n), 1), 16) - 1;
      x.from = page == ~0u ? reinterpret_cast<const uint8_t *>(&kZeros)
                           : kv.base + ((uint64_t)page * (uint32_t)kv.piece + slot * row_bytes);
    }
    return x;
  };
  // the i-th of its loads: tokens' latents, then (NI) their turned parts.  Pieces
  // past a part stay the zeros that they were.
  auto load_one = [&](const Eight &x, int i) {
    const bool turn = i == NI;
    const int at = turn ? (FP8 ? x.at & ~15 : x.at) : x.at + i * RPI;
    const int row = (at & 15) + (turn ? turn_row : lat_row);  // of the run
    const uint32_t lds = turn ? x.to + 32 * RC + at * RR : x.to + at * RC;
    const uint32_t piece =
        turn ? turn_piece ^ (turn_swap_of(at) << 4) : lat_piece ^ (swap_of(at) << 4);
    if constexpr (MODE == kPlain) {
      const uint32_t off = __umul24(min(row, x.last), row_bytes) + piece + (turn ? RC : 0);
      to_lds(lds, x.from, off & x.rows, x.there);
    } else {
      const uint8_t *p;
      if constexpr (WHOLE) {
        p = x.from +
            ((__umul24(min(row, x.last), row_bytes) + piece + (turn ? C * EB : 0)) & x.rows);
      } else {
        const uint32_t page = __shfl(load_page, x.at_n * 16 + row);
        const int slot = __shfl(load_slot, x.at_n * 16 + row);
        p = kv.base + ((uint64_t)page * (uint32_t)kv.piece + (uint32_t)slot * row_bytes +
                       (turn ? C * EB : 0) + piece);
        if (page == ~0u) p = reinterpret_cast<const uint8_t *>(&kZeros);
      }
      const uint64_t in = __ballot(piece < (uint32_t)((turn ? R : C) * EB));
      to_lds_some(lds, p, x.there,
                  (uint64_t)uniform((uint32_t)(in >> 32)) << 32 | uniform((uint32_t)in));
    }
  };

  float m = kNegInf, l = 0.f;
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  uint32_t odd = 0;

  // Places of this lane's reads in a tile: of keys, of turned parts, of values.
  // Which pieces of sixteen are read turns bits 4 to 7 of the place, which are the
  // low bits of a piece; tiles and rows are whole 256 bytes (turned parts 64, 128).
  const uint32_t key_at = c * RC + ((h ^ swap_of(c)) << 4);
  const uint32_t turn_at = 32 * RC + c * RR + ((h ^ turn_swap_of(c)) << 4);
  // of values the first sixteen tokens': those that a lane's scores are of
  const int val_row = FP8 ? (c16 >> 3) * 8 + h * 4 + ((c16 >> 1) & 3) : h * 4 + (c16 >> 2);
  const uint32_t val_at =
      val_row * RC + (c16 & 1) * 8 +
      (((FP8 ? g & 1 : (g & 1) * 2 + ((c16 >> 1) & 1)) ^ swap_of(val_row)) << 4);

  // Of the batch of runs that is computed: which pages are not there; the scales
  // of latents, times scale_log2, its logarithm (within bounds); of turned parts in
  // units of the former, which is held to 2^-60 of them for that.
  uint64_t gone_of = 0;
  float sc_of = 1.f, sc2_of = 1.f, sr_of = 1.f, log_of = 0.f;
  int n0_of = -(1 << 20);
  auto batch = [&](int step) {
    if (step * 2 - n0_of < BATCH) return;
    n0_of = step * 2 - step * 2 % BATCH;
    uint32_t page;
    int slot;
    look(n0_of, page, slot);
    gone_of = __ballot(page == ~0u);
    if (FP8) {
      const float *sp = kv.scales + (uint64_t)(page == ~0u ? 0 : page) * 2;
      float sc = sp[0], sr = sp[1];
      here(sc);
      here(sr);
      if (page == ~0u) sc = sr = 1.f;
      const float least = fmaxf(fabsf(sr) * 0x1p-60f, 0x1p-100f);
      sc_of = sc;
      if (fabsf(sc) < least) sc = sc < 0.f ? -least : least;
      sc2_of = sc * a.scale_log2;
      sr_of = sr / sc;
      log_of = __log2f(fmaxf(fabsf(sc), 0x1p-60f));
    }
  };

  // The i-th piece of a token's key that is read: the turned part's, then those
  // whose places differ by whole 256 bytes one after another; and of Q beside it.
  constexpr int KB = 8, KQ = KC / KB;  // reads of two halves of 16 pieces
  auto key_of = [](int i) { return i < KR ? KC + i : (i - KR) % KQ * KB + (i - KR) / KQ; };
  auto key_piece = [&](uint32_t tile, int i) {
    const int k = key_of(i);
    const uint32_t at = k >= KC ? (tile + turn_at) ^ ((k - KC) << 5)
                                : ((tile + key_at) ^ ((k & 7) << 5)) + (k >> 3) * 256;
    return *reinterpret_cast<lds_u32x4 *>(at);
  };
  // Values of sixteen tokens: a lane's eight of them for each of 32 elements.
  struct Values {
    u32x2 w[FP8 ? 1 : 2];
  };
  auto value_piece = [&](uint32_t run, int dt) {
    Values v;
    if constexpr (FP8) {
      const uint32_t at = ((run + val_at) ^ ((dt & 7) << 5)) + (dt >> 3) * 256;
      v.w[0] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                             reinterpret_cast<lds_i32x2 *>(at)));
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {  // eight tokens on
        const uint32_t at = ((run + val_at) ^ ((dt & 3) << 6 | (swap_of(8) << 4) * j)) +
                            (dt >> 2) * 256 + j * 8 * RC;
        v.w[j] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                               reinterpret_cast<lds_s16x4 *>(at)));
      }
    }
    return v;
  };

  // Zeros in place of a tile's values that are not finite, once every wave that
  // shares it has read its keys.
  auto mend = [&](int step) {
    if (QW > 1) __syncthreads();
    uint8_t *p = ring + (step % NST) * STAGE + kg * TILE + qg * (32 / QW) * RC + lane * 16;
#pragma unroll 1
    for (int i = 0; i < 32 / QW * RC / 1024; ++i) {
      u32x4 v = *reinterpret_cast<u32x4 *>(p + i * 1024);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t bad = odd_mask<ACT, FP8>(v[j]);
        odd |= bad;
        v[j] &= ~bad;
      }
      *reinterpret_cast<u32x4 *>(p + i * 1024) = v;
    }
    if (QW > 1) __syncthreads();
    else wait_reads();
  };

  // ---- a tile's scores, S^T = K Q^T: column c, tokens (i / 4) * 8 + h * 4 +
  // i % 4; beside each read's products something else, side(i).  fp8: the turned
  // part's come first and go into units of the latents' scale.
  f32x16 x;
  auto scores = [&](int step, auto side) {
    const uint32_t tile = ring_at + (step % NST) * STAGE + kg * TILE;
    u32x4 w[AHEAD + 1];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) w[i] = key_piece(tile, i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < KN; ++i) {
      if (i + AHEAD < KN) w[(i + AHEAD) % (AHEAD + 1)] = key_piece(tile, i + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
      const u32x4 v = w[i % (AHEAD + 1)];
      if constexpr (FP8) {
        const u32x4 lo = {fp8_pair<ACT, false>(v[0]), fp8_pair<ACT, true>(v[0]),
                          fp8_pair<ACT, false>(v[1]), fp8_pair<ACT, true>(v[1])};
        const u32x4 hi = {fp8_pair<ACT, false>(v[2]), fp8_pair<ACT, true>(v[2]),
                          fp8_pair<ACT, false>(v[3]), fp8_pair<ACT, true>(v[3])};
        if (i == 0) multiply32<ACT, true>(x, lo, qreg[2 * key_of(i)]);
        else multiply32<ACT, false>(x, lo, qreg[2 * key_of(i)]);
        multiply32<ACT, false>(x, hi, qreg[2 * key_of(i) + 1]);
        if (i == KR - 1) {
          settled(x);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int n = step * 2 + (j >> 3) - n0_of;
            x[j] *= WHOLE ? of_lane(sr_of, n)
                          : __shfl(sr_of, n * 16 + (j >> 2 & 1) * 8 + h * 4 + (j & 3));
          }
        }
      } else {
        if (i == 0) multiply32<ACT, true>(x, v, qreg[key_of(i)]);
        else multiply32<ACT, false>(x, v, qreg[key_of(i)]);
      }
      side(i);
      __builtin_amdgcn_sched_barrier(0);
    }
    settled(x);
  };

  // ---- its weights, masked
  float y[16], vs[FP8 ? 16 : 1];
  float ls[2] = {0.f, 0.f};
  auto mask = [&](int step) {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i];
    const int n = step * 2 - n0_of, tok0 = run_at(step * 2);
    if constexpr (FP8) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = n + (i >> 3), at = r * 16 + (i >> 2 & 1) * 8 + h * 4 + (i & 3);
        y[i] *= WHOLE ? of_lane(sc2_of, r) : __shfl(sc2_of, at);
        vs[i] = WHOLE ? of_lane(sc_of, r) : __shfl(sc_of, at);
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) ls[r] = WHOLE ? of_lane(log_of, n + r) : 0.f;
    }
    const uint32_t gone = WHOLE ? ((gone_of >> n) & 1 ? 0xffffu : 0u) |
                                      ((gone_of >> (n + 1)) & 1 ? 0xffff0000u : 0u)
                                : (uint32_t)(gone_of >> (n * 16));
    if (gone || tok0 + 32 > all_lim) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = (i >> 2) * 8 + h * 4 + (i & 3);
        const bool out = tok0 + at >= lim || ((gone >> at) & 1);
        y[i] = out ? kNegInf : y[i];
        // (a scale that is not finite, or one of a block that the row sees
        // nothing of)
        if (FP8) vs[i] = out ? 0.f : vs[i];
      }
    }
  };
  // The weights in kSides pieces of about the same work, to stand between
  // products.  The reference counts a value's scale in, within bounds, so that its
  // weight with the scale fits 16 bits.
  constexpr int kSides = 28;
  const float of_score = FP8 ? 1.f : a.scale_log2;
  float top, f, ref;
  uint64_t jump = 0;
  u32x4 ph[2];
  auto weigh = [&](int i) {
    if (i == 0 || i == 1) {
      float t = kNegInf;
#pragma unroll
      for (int j = i * 8; j < i * 8 + 8; ++j) {
        if constexpr (FP8 && !WHOLE) t = fmaxf(t, y[j] + __log2f(fmaxf(fabsf(vs[j]), 0x1p-60f)));
        else t = fmaxf(t, y[j]);
      }
      if constexpr (FP8 && WHOLE) t += ls[i];
      top = i == 0 ? t : fmaxf(top, t);
    } else if (i == 2) {
      top = max_rows32(top) * of_score;
    } else if (i == 3) {
      const bool over = top > m + kSlack;
      jump = __ballot(over);
      top = over ? top : m;
      f = m == kNegInf ? 0.f : exp2_fast(m - top);
      l *= f;
      m = top;
      ref = m == kNegInf ? 0.f : m - kShift;
    } else {
      const int j = (i - 4) / 3, part = (i - 4) % 3;  // pair j of values
      if (part < 2) {
        float &p = y[2 * j + part];
        p = exp2_fast(p * of_score - ref);
        l += p;
        if constexpr (FP8) p *= vs[2 * j + part];
      } else {
        const uint32_t w = pack_act<PV>(y[2 * j], y[2 * j + 1]);
        ph[j >> 2][j & 3] = w;
        if constexpr (TWO) {  // the first bf16, or zeros, taken off
          const uint32_t lo = __builtin_amdgcn_perm(w, w, second ? 0x01000c0cu : 0x0c0c0c0cu);
          const uint32_t hi = __builtin_amdgcn_perm(w, w, second ? 0x03020c0cu : 0x0c0c0c0cu);
          ph[j >> 2][j & 3] = pack_act<kBf16>(y[2 * j] - __uint_as_float(lo),
                                              y[2 * j + 1] - __uint_as_float(hi));
        }
      }
    }
  };
  // ---- O^T += V^T P^T of sixteen tokens, loads of later ones between the products
  Values vw[VAHEAD + 1];
  auto values_ahead = [&](uint32_t run) {
#pragma unroll
    for (int n = 0; n < VAHEAD; ++n) vw[n] = value_piece(run, tile_of_sum(n));
  };
  auto add_values = [&](uint32_t run, int half, auto side) {
#pragma unroll
    for (int n = 0; n < DT; ++n) {
      if (n + VAHEAD < DT)
        vw[(n + VAHEAD) % (VAHEAD + 1)] = value_piece(run, tile_of_sum(n + VAHEAD));
      __builtin_amdgcn_sched_barrier(0);
      const Values v = vw[n % (VAHEAD + 1)];
      u32x4 af;
      if constexpr (FP8)
        af = u32x4{fp8_pair<PV, false>(v.w[0][0]), fp8_pair<PV, true>(v.w[0][0]),
                   fp8_pair<PV, false>(v.w[0][1]), fp8_pair<PV, true>(v.w[0][1])};
      else
        af = u32x4{v.w[0][0], v.w[0][1], v.w[1][0], v.w[1][1]};
      f32x16 &to = o[tile_of_sum(n)];
      to = mfma32<PV>(af, ph[half], to);
      side(n);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // ---- the ring.  With room for three steps or more, a tile's scores are made
  // beside the weights of the one before it, and loads go on all the time, NST - 1
  // steps ahead.  With room for two, sixteen tokens' place is loaded into once their
  // values have been used.  Loads stand between products: the way to LDS takes 64
  // bytes a cycle of all waves, and one that waits for it holds up its wave.  Steps
  // past the last load nothing, and what is made of their tokens goes unused.
  if (MODE != kPlain) {  // pieces past a token's parts
    for (int i = threadIdx.x * 16; i < NST * STAGE; i += kThreads * 16)
      *reinterpret_cast<u32x4 *>(ring + i) = u32x4{0, 0, 0, 0};
    __syncthreads();
  }
  auto meet = [&] {  // all waves have read what they wanted of the ring
    wait_reads();
    if (QW > 1) __syncthreads();
  };
  if (n_steps > 0) {
    constexpr int FIRST = PIPE ? NST - 1 : 2;  // steps that load before the first
    batch(0);
#pragma unroll 1
    for (int step = 0; step < FIRST; ++step)
#pragma unroll
      for (int e = 0; e < EIGHTS; ++e) {
        const Eight from = eight_of(step, e);
#pragma unroll
        for (int i = 0; i <= NI; ++i) load_one(from, i);
      }
    if (FIRST <= n_steps) wait_loads<(FIRST - 1) * LOADS>();
    else wait_loads<0>();
    if (QW > 1) __syncthreads();
    scores(0, [](int) {});
#pragma unroll 1
    for (int step = 0; step < n_steps; ++step) {
      const uint32_t tile = ring_at + (step % NST) * STAGE + kg * TILE;
      // where rows attend to different tokens, values that are not finite count as
      // zero and are left for the end
      const int first = p0 + step * STEP;
      if (all_lim < end && first + STEP > all_lim) mend(step);
      mask(step);
      batch(step + 1);
      Eight from[EIGHTS];
      // loads in even distances over `of` places
      auto load_at = [&](int at, int of, int i0, int count) {
#pragma unroll
        for (int i = 0; i < count; ++i)
          if ((2 * i + 1) * of / (2 * count) == at)
            load_one(from[(i0 + i) / (NI + 1)], (i0 + i) % (NI + 1));
      };
      constexpr int EACH = (kSides + KN - 1) / KN;
      if constexpr (PIPE) {
        // (no more loads than these are on their way while there are steps to load)
        if (step + NST - 2 < n_steps) wait_loads<(PIPE ? NST - 3 : 0) * LOADS>();
        else wait_loads<0>();
        meet();
#pragma unroll
        for (int e = 0; e < EIGHTS; ++e) from[e] = eight_of(step + NST - 1, e);
        scores(step + 1, [&](int k) {
#pragma unroll
          for (int i = 0; i < EACH; ++i)
            if (k * EACH + i < kSides) weigh(k * EACH + i);
          load_at(k, KN, 0, LOADS / 2);
          if (k == KN - 2) values_ahead(tile);
        });
        if (jump) rescale(o, f);
        add_values(tile, 0, [&](int n) { load_at(n, 2 * DT, LOADS / 2, LOADS - LOADS / 2); });
        values_ahead(tile + 16 * RC);
        add_values(tile + 16 * RC, 1,
                   [&](int n) { load_at(DT + n, 2 * DT, LOADS / 2, LOADS - LOADS / 2); });
      } else {
        constexpr int HALF = LOADS / 2;
        values_ahead(tile);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kSides; ++i) weigh(i);
        if (jump) rescale(o, f);
        add_values(tile, 0, [](int) {});
        values_ahead(tile + 16 * RC);
        meet();
#pragma unroll
        for (int e = 0; e < EIGHTS; ++e) from[e] = eight_of(step + 2, e);
        add_values(tile + 16 * RC, 1, [&](int n) { load_at(n, DT, 0, HALF); });
        if (step + 2 < n_steps) wait_loads<HALF>();
        else wait_loads<0>();
        meet();
        scores(step + 1, [&](int k) { load_at(k, KN, HALF, HALF); });
      }
    }
    wait_loads<0>();
  }
  // ---- values that are not finite, where not every row attends to them: a
  // weight that is not zero made the whole row NaN, zero times them is NaN too
  if (!FP8 && __syncthreads_or(odd != 0)) {
    asm volatile("s_nop 15\n\ts_nop 7" : : : "memory");  // as in rescale()
    const int last = min(p0 + part_steps * STEP, end);
    for (int at = max(all_lim & ~(STEP - 1), p0); at < last; ++at) {
      const int e = over_page(kv, at);
      const uint32_t page = table[e];
      if (page >= (uint32_t)kv.num_pages) continue;
      const uint16_t *p = reinterpret_cast<const uint16_t *>(
          kv.base + ((uint64_t)page * (uint32_t)kv.piece + (uint32_t)(at - e * T) * row_bytes));
      const bool sees = at < lim && (at - p0) / 32 % KG == kg;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const int d = dt * 32 + i4 * 8 + h * 4;
          const u32x2 w = *reinterpret_cast<const u32x2 *>(p + (d < C ? d : 0));
          const uint32_t bad[2] = {odd_mask<ACT, false>(w[0]), odd_mask<ACT, false>(w[1])};
          float add[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            add[i] = d < C && sees && (bad[i >> 1] >> (16 * (i & 1)) & 0xffff)
                         ? __uint_as_float(0x7fc00000u)
                         : 0.f;
          add4(o[dt], i4, add);
        }
        __builtin_amdgcn_sched_barrier(0);  // a block's loads at a time: registers
      }
    }
  }

  // ---- the groups' sums become one: the rows' output, or a part of it, which
  // lies as the registers do, [32 rows][tile of 32 elements][i4][lane]
  const float total_of = add_rows32(l);
  const float ref_of = m == kNegInf ? kNegInf : m - kShift;
  const int cols = (C + 31) & ~31;
  float *part_of = a.parts + (int64_t)blockIdx.x * (QW * 32) * (cols + 2);
  const int64_t row = sq.row0 + my_q, head = my - my_q * HQ;
  auto emit = [&](int dt, int i4, const f32x4 &v, float norm) {
    const int d = dt * 32 + i4 * 8 + h * 4;
    if (!mine || d >= C) return;
    if (parts == 1)
      *reinterpret_cast<u32x2 *>(a.out.data + row * a.out.row_stride + head * a.out.head_stride +
                                 d) =
          u32x2{pack_act<ACT>(v[0] * norm, v[1] * norm), pack_act<ACT>(v[2] * norm, v[3] * norm)};
    else
      *reinterpret_cast<f32x4 *>(part_of + cg * 32 * cols +
                                 ((dt * 4 + i4) * kLanes + lane) * 4) = v;
  };
  auto emit_statistics = [&](float ref, float total) {
    if (!mine || h) return;
    if (parts > 1)
      *reinterpret_cast<f32x2 *>(part_of + QW * 32 * cols + 2 * (qg * 32 + c)) = f32x2{ref, total};
    else if (a.lse)
      a.lse[row * HQ + head] =
          total == 0.f ? kNegInf : (ref + __log2f(total)) * 0.6931471805599453f;
  };
  if (a.slices > 0 && part == 0 && threadIdx.x == 0) {  // for the join
    a.units[2 * ((int64_t)s * a.tiles_most + r0 / (QW * 32))] = blockIdx.x;
    a.units[2 * ((int64_t)s * a.tiles_most + r0 / (QW * 32)) + 1] = parts;
  }
  if constexpr (KG == 1) {
    const float norm = total_of == 0.f ? 0.f : 1.f / total_of;
    auto tile_of_o = [&](int dt, int i4) {
      return f32x4{o[dt][i4 * 4], o[dt][i4 * 4 + 1], o[dt][i4 * 4 + 2], o[dt][i4 * 4 + 3]};
    };
    if constexpr (TWO) {  // both waves of a column have half of its tiles' sums to join
      constexpr int HALF = DT / 2;
      static_assert(kWaves * HALF * 4 * kLanes * 16 <= BYTES, "every wave's other half");
      f32x4 *sums = reinterpret_cast<f32x4 *>(ring) + lane;
      auto give = [&](int first) {
#pragma unroll
        for (int dt = 0; dt < HALF; ++dt) {
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4)
            sums[((wave * HALF + dt) * 4 + i4) * kLanes] = tile_of_o(first + dt, i4);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      auto take = [&](int first) {
#pragma unroll
        for (int dt = 0; dt < HALF; ++dt) {
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4)
            emit(first + dt, i4,
                 tile_of_o(first + dt, i4) + sums[(((wave ^ 2) * HALF + dt) * 4 + i4) * kLanes],
                 norm);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      __syncthreads();  // the ring has been read
      if (second) give(0);
      else give(HALF);
      __syncthreads();
      if (second) {
        take(HALF);
        return;
      }
      take(0);
    } else {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) emit(dt, i4, tile_of_o(dt, i4), norm);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    emit_statistics(ref_of, total_of);
  } else {
    if (h == 0) {
      wave_ml[wave][c][0] = ref_of;
      wave_ml[wave][c][1] = total_of;
    }
    __syncthreads();  // and the ring has been read
    float ref = kNegInf, total = 0.f;
#pragma unroll
    for (int k = 0; k < KG; ++k) ref = fmaxf(ref, wave_ml[k * QW + qg][c][0]);
    const float zero = ref == kNegInf ? 0.f : ref;
#pragma unroll
    for (int k = 0; k < KG; ++k)
      total += exp2_fast(wave_ml[k * QW + qg][c][0] - zero) * wave_ml[k * QW + qg][c][1];
    const float f = ref_of == kNegInf ? 0.f : exp2_fast(ref_of - zero);
    const float norm = total == 0.f ? 0.f : 1.f / total;
    constexpr int RD = CR / 32;
    f32x4 *sums = reinterpret_cast<f32x4 *>(ring);
#pragma unroll
    for (int round = 0; round < 2; ++round) {
      if (round) __syncthreads();
#pragma unroll
      for (int d = 0; d < RD; ++d)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const int dt = round * RD + d;
          sums[((wave * RD + d) * 4 + i4) * kLanes + lane] =
              f32x4{o[dt][i4 * 4] * f, o[dt][i4 * 4 + 1] * f,
                    o[dt][i4 * 4 + 2] * f, o[dt][i4 * 4 + 3] * f};
        }
      __syncthreads();
      for (int d = kg; d < RD; d += KG)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < KG; ++k)
            v += sums[(((k * QW + qg) * RD + d) * 4 + i4) * kLanes + lane];
          emit(round * RD + d, i4, v, norm);
        }
    }
    if (kg == 0) emit_statistics(ref, total);
  }
}

// Joins the parts of a unit's 32 rows, some pieces (a quarter of a tile's 32
// elements) of them:
//   o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i,  m = max_i m_i.
// A launch of its own, so that many workgroups read the parts and nothing waits
// or counts (joined by the last of a unit's workgroups, 24 sequences of 2-4 rows took
// 152 us in place of 89).  256 parts of 128 rows: 19 us (67 MB, 3.5 TB/s); 5 parts of each of 64
// sequences: 8 us.  A wave runs once over a piece's parts, kAhead at a time, with the
// running reference and sums of a softmax; where there are many, over every
// kGroups-th, and then the waves' become one.
constexpr int kGroups = 8, kJoinThreads = kGroups * kLanes, kAhead = 8;
template <int ACT>
__global__ __launch_bounds__(kJoinThreads) void join_latent(LatentAttendArgs a) {
  __shared__ f32x4 sums[kGroups][kLanes];
  __shared__ f32x2 stats[kGroups][kLanes];
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int g = uniform((int)threadIdx.x >> 6);
  const int QW = a.wave_columns, HQ = a.q_heads, C = a.latent, cols = (C + 31) & ~31;
  uint32_t u = blockIdx.x;
  const int slice = u % a.slices;
  u /= a.slices;
  const int qg = u % QW;
  u /= QW;
  const int tile = u % a.tiles_most, s = u / a.tiles_most;
  const Seq sq = sequence(a.b, s);
  const int r = tile * QW * 32 + qg * 32 + c, rows_all = sq.rows * HQ;
  if (r - c >= rows_all) return;
  const int w0 = a.units[2 * ((int64_t)s * a.tiles_most + tile)];
  const int parts = a.units[2 * ((int64_t)s * a.tiles_most + tile) + 1];
  // (with starts of rows that decrease there are more units than the host counts and
  // launches, and nobody writes this for the last of them)
  if (parts <= 1 || parts > a.split_grid || w0 < 0 || w0 > a.split_grid - parts) return;
  const int64_t pitch = (int64_t)(QW * 32) * (cols + 2);
  const float *first = a.parts + (int64_t)w0 * pitch;
  const float *ml = first + QW * 32 * cols + 2 * (qg * 32 + c);
  const bool alone = parts <= 2 * kAhead;
  const int k_first = alone ? 0 : g, k_step = alone ? 1 : kGroups;
  const int pieces = a.slices * (alone ? kGroups : 1);
  for (int piece = alone ? slice * kGroups + g : slice; piece < cols / 8; piece += pieces) {
    const int d = piece * 8 + h * 4;
    const bool mine = r < rows_all && d < C;
    const float *p = first + qg * 32 * cols + (piece * kLanes + lane) * 4;
    float m = kNegInf, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = k_first; k0 < parts; k0 += k_step * kAhead) {
      f32x2 of[kAhead];
      f32x4 v[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int k = k0 + i * k_step;
        of[i] = f32x2{kNegInf, 0.f};
        v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (mine && k < parts) {
          of[i] = *reinterpret_cast<const f32x2 *>(ml + k * pitch);
          v[i] = *reinterpret_cast<const f32x4 *>(p + k * pitch);
        }
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) top = fmaxf(top, of[i][0]);
      const float ref = top == kNegInf ? 0.f : top, f = exp2_fast(m - ref);
      m = top;
      l *= f;
      acc *= f;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const float w = exp2_fast(of[i][0] - ref);
        l += w * of[i][1];
        acc += w * v[i];
      }
    }
    if (!alone) {
      sums[g][lane] = acc;
      stats[g][lane] = f32x2{m, l};
      __syncthreads();
      if (g == 0) {
        m = kNegInf;
#pragma unroll
        for (int k = 0; k < kGroups; ++k) m = fmaxf(m, stats[k][lane][0]);
        const float ref = m == kNegInf ? 0.f : m;
        l = 0.f;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
          const float w = exp2_fast(stats[k][lane][0] - ref);
          l += w * stats[k][lane][1];
          acc += w * sums[k][lane];
        }
      }
      __syncthreads();
    }
    if (mine && (alone || g == 0)) {
      const float norm = l == 0.f ? 0.f : 1.f / l;
      const int64_t row = sq.row0 + r / HQ, head = r % HQ;
      *reinterpret_cast<u32x2 *>(a.out.data + row * a.out.row_stride + head * a.out.head_stride +
                                 d) =
          u32x2{pack_act<ACT>(acc[0] * norm, acc[1] * norm),
                pack_act<ACT>(acc[2] * norm, acc[3] * norm)};
      if (d == 0 && a.lse)
        a.lse[row * HQ + head] = l == 0.f ? kNegInf : (m + __log2f(l)) * 0.6931471805599453f;
    }
  }
}

void go(void (*kernel)(LatentAttendArgs), const LatentAttendArgs &a, hipStream_t s) {
  hipLaunchKernelGGL(kernel, dim3((unsigned)a.split_grid), dim3(kThreads), 0, s, a);
}

template <int ACT, bool FP8, int CT, Mode MODE>
hipError_t columns(const LatentAttendArgs &a, hipStream_t s) {
  if constexpr (FP8) {
    if (a.wave_columns == 1) go(attend_latent<ACT, true, CT, 1, MODE, false>, a, s);
    if (a.wave_columns == 2) go(attend_latent<ACT, true, CT, 2, MODE, false>, a, s);
  }
  constexpr bool BF16 = ACT == kBf16 && !FP8;
  if constexpr (BF16)
    if (a.two_weights) go(attend_latent<ACT, false, CT, 4, MODE, true>, a, s);
  if (a.wave_columns == 4 && !(BF16 && a.two_weights))
    go(attend_latent<ACT, FP8, CT, 4, MODE, false>, a, s);
  if (a.slices > 0)
    hipLaunchKernelGGL(join_latent<ACT>,
                       dim3((unsigned)a.b.n_seqs * a.tiles_most * a.wave_columns * a.slices),
                       dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

template <int ACT, bool FP8, int CT>
hipError_t rows(const LatentAttendArgs &a, hipStream_t s) {
  if (a.kv.page_tokens % 16 != 0) return columns<ACT, FP8, CT, kPages>(a, s);
  if (a.latent != CT || a.turn != kTurn) return columns<ACT, FP8, CT, kRows>(a, s);
  return columns<ACT, FP8, CT, kPlain>(a, s);
}

template <int ACT, bool FP8>
hipError_t latents(const LatentAttendArgs &a, hipStream_t s) {
  return a.latent <= 256 ? rows<ACT, FP8, 256>(a, s) : rows<ACT, FP8, 512>(a, s);
}

}  // namespace

hipError_t launch_attend_latent(const LatentAttendArgs &a, int act, int fp8, hipStream_t s) {
  (void)hipGetLastError();
  if (act == kBf16) return fp8 ? latents<kBf16, true>(a, s) : latents<kBf16, false>(a, s);
  return fp8 ? latents<kF16, true>(a, s) : latents<kF16, false>(a, s);
}

}  // namespace ea
