// Pages from place to place in a cache: whole pages copied in every layer, and
// tokens of edited contexts moved together into other pages, their keys turned
// from the old position to the new one.
//
// What bounds both is memory: each byte is read once and written once.
//
// Copies: a wave takes 4 KiB, with all its loads on their way before the first
// store, and pieces of planes go by units of their own in the same launch.  4,096
// pages of 12 layers, fp8 with bounds, 1.72 GB: 360 us (4.75 TB/s, as a large
// library copy).
//
// Moves: a wave takes a block's 16 tokens, whose places and angles it looks up once
// for all heads and several layers.  16 contexts of 8,192-65,536 tokens, fp8 with
// bounds, two layers, 1.71 GB: 420 us (4.06 TB/s); a wave for each head and layer,
// with the lookups each time: 1,902 us.  Beside the reading a wave decodes, searches a
// block's largest value, rounds and makes bounds: 15% below the copies' rate.
#include <hip/hip_runtime.h>

#include "ea_kv_blocks.hpp"
#include "ea_kv_device.hpp"

namespace ea {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kLanes;
constexpr int kLoads = 4;                        // 16-byte loads of a lane
constexpr int64_t kRun = kLoads * kLanes * 16;   // bytes of a piece that a wave copies

// `bytes` from src to dst by a wave, words of `W` bytes.
template <typename W>
__device__ inline void copy_words(uint8_t *dst, const uint8_t *src, int64_t bytes, int lane) {
  for (int64_t i = lane * (int64_t)sizeof(W); i < bytes; i += kLanes * sizeof(W))
    *reinterpret_cast<W *>(dst + i) = *reinterpret_cast<const W *>(src + i);
}

__global__ __launch_bounds__(kThreads) void copy_pages(CopyArgs a, int64_t runs, int64_t units) {
  const int lane = threadIdx.x & 63;
  int64_t u = (int64_t)blockIdx.x * kWaves + uniform((int)threadIdx.x >> 6);
  if (u >= units) return;
  const bool planes = u >= runs;
  if (planes) u -= runs;
  const int per = planes ? 1 : a.runs_piece;
  const int run = u % per;
  u /= per;
  const int layer = u % a.layers, i = u / a.layers;
  const int src = a.src[i], dst = a.dst[i];
  if ((uint32_t)src >= (uint32_t)a.num_pages || (uint32_t)dst >= (uint32_t)a.num_pages) return;
  const int64_t from = (int64_t)layer * a.num_pages + src, to = (int64_t)layer * a.num_pages + dst;
  if (!planes) {
    const int64_t at = run * kRun + lane * 16;
    const u32x4 *p = reinterpret_cast<const u32x4 *>(a.base + from * a.piece + at);
    u32x4 *q = reinterpret_cast<u32x4 *>(a.base + to * a.piece + at);
    u32x4 v[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (at + k * (kRun / kLoads) < a.piece) v[k] = p[k * kLanes];
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (at + k * (kRun / kLoads) < a.piece) q[k * kLanes] = v[k];
    return;
  }
#pragma unroll
  for (int k = 0; k < kCopyPlanes; ++k) {
    uint8_t *b = a.plane[k];
    if (!b) continue;
    const int64_t n = a.plane_bytes[k];
    uint8_t *q = b + to * n;
    const uint8_t *p = b + from * n;
    if (((n | (uintptr_t)b) & 7) == 0) copy_words<u32x2>(q, p, n, lane);
    else if (((n | (uintptr_t)b) & 3) == 0) copy_words<uint32_t>(q, p, n, lane);
    else copy_words<uint8_t>(q, p, n, lane);
  }
}

// Elements of a stored head beside the ones that a lane holds, for the ways of
// pairing whose halves are no whole pieces: x turned by |position| `at`.
template <int ACT, bool FP8>
__device__ inline void turn_apart(const uint8_t *head, const Place &p, const float *rope, int at,
                                  float sign, int dim, bool interleaved, float x[16]) {
#pragma clang fp contract(off)
  const int half = dim >> 1;
  const float *cs = rope + (int64_t)at * dim, *sn = cs + half;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    if (!p.in[n] || p.d[n] >= dim) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = p.d[n] + i;
      if (d >= dim) break;
      const bool upper = interleaved ? d & 1 : d >= half;
      const int f = interleaved ? d >> 1 : upper ? d - half : d;
      const int e = interleaved ? d ^ 1 : upper ? d - half : d + half;
      float y;
      if constexpr (FP8) y = __builtin_amdgcn_cvt_pk_f32_fp8(head[e], false)[0];
      else y = act_to_float<ACT>(reinterpret_cast<const uint16_t *>(head)[e]);
      const float xc = x[n * 8 + i] * cs[f], ys = y * (sn[f] * sign);
      x[n * 8 + i] = upper ? xc + ys : xc - ys;
    }
  }
}

// One wave: one block in some layers, all KV heads, keys and values.  Where its
// tokens are, and the angles that they turn by, serve all of them; the next
// head's elements load while this one's are turned and written.  HALVES: the
// turn, if any, pairs whole pieces of 8.  ONE: a block is 16 tokens at most,
// which registers hold; otherwise the ones after them are read again for each
// use.
template <int ACT, bool FP8, int LP, bool HALVES, bool ONE>
__global__ __launch_bounds__(kThreads) void move_tokens(MoveArgs a, uint32_t units) {
  constexpr int EB = FP8 ? 1 : 2, TW = kLanes / LP;  // tokens of a pass
  constexpr int KEEP = 16 / TW;  // passes whose tokens stay in registers
  constexpr int W = FP8 ? 2 : 4;  // words of 8 elements
  const int lane = threadIdx.x & 63;
  uint32_t u = blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  if (u >= units) return;
  const int j = u % a.blocks_most;
  u /= a.blocks_most;
  const int s = u % a.n_seqs, layer0 = u / a.n_seqs * a.layers_wave;
  const int layer1 = min(layer0 + a.layers_wave, a.layers);
  const MovedBlock m = moved_block(a, s, j);
  if (m.n <= 0) return;
  const int H = a.kv.heads, D = a.kv.head_dim;
  const uint32_t token_bytes = H * D * EB, half_piece = (uint32_t)(a.kv.piece >> 1);
  const int t0 = lane / LP;
  const bool with_bounds = a.kv.bounds != nullptr;
  const Place at = place_of(lane % LP, D, a.rope != nullptr, a.rope_dim, a.interleaved);

  MovedToken tok[KEEP];
  Angles an[KEEP];
  auto angles = [&](const MovedToken &t) {
    Angles g = {};
    if (HALVES && t.by != 0) g = angles_of(a.rope, abs(t.by), a.rope_dim, at);
    if (t.by < 0) {
      g.s[0] = -g.s[0];
      g.s[1] = -g.s[1];
    }
    return g;
  };
#pragma unroll
  for (int k = 0; k < KEEP; ++k) {
    tok[k] = {-1, 0, 0};
    if (t0 + k * TW < m.n) tok[k] = moved_token(a, m, t0 + k * TW);
    an[k] = angles(tok[k]);
  }

  for (int layer = layer0; layer < layer1; ++layer) {
    KvLayer kv = a.kv;
    kv.base += layer * a.layer_bytes;
    if (FP8) kv.scales += layer * a.layer_scales;
    if (with_bounds) {
      kv.bounds += (int64_t)layer * kv.num_pages * 2 * H * D;
      kv.bound_scales += (int64_t)layer * kv.num_pages * H;
    }
    // planes: keys of head plane / 2, then its values
    auto head_at = [&](int plane) { return (plane & 1 ? half_piece : 0) + (plane >> 1) * D * EB; };
    struct Raw {
      uint32_t w[2][W];
      float scale;
    };
    auto load = [&](const MovedToken &t, int plane) {
      Raw r = {};
      r.scale = 1.f;
      if (t.page < 0) return r;
      const uint8_t *p = kv.base + ((uint64_t)t.page * kv.piece + t.slot * token_bytes +
                                    head_at(plane));
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        if (!at.in[n]) continue;
        if constexpr (FP8) {
          const u32x2 v = *reinterpret_cast<const u32x2 *>(p + at.d[n]);
          r.w[n][0] = v[0];
          r.w[n][1] = v[1];
        } else {
          const u32x4 v = *reinterpret_cast<const u32x4 *>(p + at.d[n] * 2);
#pragma unroll
          for (int i = 0; i < 4; ++i) r.w[n][i] = v[i];
        }
      }
      if (FP8)
        r.scale = kv.scales[(int64_t)t.page * kv.scale_page + (plane & 1 ? kv.scale_kv : 0) +
                            (plane >> 1) * kv.scale_head];
      return r;
    };
    // Elements as stored (fp8: codes, their scale apart), turned.
    auto values = [&](const Raw &r, const MovedToken &t, const Angles &g, int plane, float x[16]) {
#pragma clang fp contract(off)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        if constexpr (FP8) {
          fp8_values(r.w[n][0], x + n * 8);
          fp8_values(r.w[n][1], x + n * 8 + 4);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            x[n * 8 + i] = act_to_float<ACT>((uint16_t)(r.w[n][i >> 1] >> (16 * (i & 1))));
        }
      }
      if ((plane & 1) || t.by == 0) return;
      if constexpr (HALVES) {
        if (at.paired) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float co = g.c[i >> 2][i & 3], si = g.s[i >> 2][i & 3], y = x[i], z = x[8 + i];
            const float yc = y * co, zs = z * si, zc = z * co, ys = y * si;
            x[i] = yc - zs;
            x[8 + i] = zc + ys;
          }
        }
      } else {
        turn_apart<ACT, FP8>(kv.base + ((uint64_t)t.page * kv.piece + t.slot * token_bytes +
                                        head_at(plane)),
                             at, a.rope, abs(t.by), t.by < 0 ? -1.f : 1.f, a.rope_dim,
                             a.interleaved, x);
      }
    };
    // of a token that no register holds
    auto fetch = [&](int i, int plane, float x[16]) {
      const MovedToken t = moved_token(a, m, i);
      const Raw r = load(t, plane);
      values(r, t, angles(t), plane, x);
      return r.scale;
    };

    Raw next[KEEP];
#pragma unroll
    for (int k = 0; k < KEEP; ++k) next[k] = load(tok[k], 0);
    for (int plane = 0; plane < 2 * H; ++plane) {
      const bool value = plane & 1, bounds = !value && with_bounds;
      const int h = plane >> 1;
      uint8_t *dst = kv.base + ((uint64_t)m.page * kv.piece + head_at(plane));
      if constexpr (!FP8) {  // nothing of values changes
        if (value) {
          Raw now[KEEP];
#pragma unroll
          for (int k = 0; k < KEEP; ++k) {
            now[k] = next[k];
            if (plane + 1 < 2 * H) next[k] = load(tok[k], plane + 1);
          }
          auto put = [&](int t, const Raw &r) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
              if (at.in[n])
                *reinterpret_cast<u32x4 *>(dst + t * token_bytes + at.d[n] * 2) =
                    u32x4{r.w[n][0], r.w[n][1], r.w[n][2], r.w[n][3]};
          };
#pragma unroll
          for (int k = 0; k < KEEP; ++k)
            if (t0 + k * TW < m.n) put(t0 + k * TW, now[k]);
          if constexpr (!ONE)
            for (int t = t0 + KEEP * TW; t < m.n; t += TW) put(t, load(moved_token(a, m, t), plane));
          continue;
        }
      }
      float x[KEEP][16], scales[KEEP];
#pragma unroll
      for (int k = 0; k < KEEP; ++k) {
        values(next[k], tok[k], an[k], plane, x[k]);
        scales[k] = next[k].scale;
        if (plane + 1 < 2 * H) next[k] = load(tok[k], plane + 1);
      }
      float scale = 1.f, inv = 1.f;
      if constexpr (FP8) {
        // of all values first: max passes over NaN, and infinities are rare
        auto largest = [&](const float y[16], float by) {
          float v = 0.f;
#pragma unroll
          for (int i = 0; i < 16; i += 2) v = fmaxf(fmaxf(v, fabsf(y[i])), fabsf(y[i + 1]));
          return v * fabsf(by);
        };
        auto largest_finite = [&](const float y[16], float by) {
          float v = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) v = fmaxf(v, finite(y[i] * by) ? fabsf(y[i] * by) : 0.f);
          return v;
        };
        auto over = [&](auto of) {
          float v = 0.f;
#pragma unroll
          for (int k = 0; k < KEEP; ++k) v = fmaxf(v, of(x[k], scales[k]));  // zeros past the last
          if constexpr (!ONE)
            for (int t = t0 + KEEP * TW; t < m.n; t += TW) {
              float y[16];
              const float by = fetch(t, plane, y);
              v = fmaxf(v, of(y, by));
            }
          return max_wave(v);
        };
        float amax = over(largest);
        if (!finite(amax)) amax = over(largest_finite);
        scale = fp8_scale(amax);
        inv = power_inverse(scale);
        if (lane == 0)
          kv.scales[(int64_t)m.page * kv.scale_page + (value ? kv.scale_kv : 0) +
                    h * kv.scale_head] = scale;
      }
      float lo[16], hi[16];
      if (bounds) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          lo[i] = __builtin_inff();
          hi[i] = kNegInf;
        }
      }
      auto store = [&](int t, float y[16], float by) {
        const float f = factor_of(by, inv);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          if (!at.in[n]) continue;
          uint8_t *q = dst + t * token_bytes + at.d[n] * EB;
          float z[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = FP8 ? y[n * 8 + i] * f : y[n * 8 + i];
          if constexpr (FP8) {
            const u32x2 w = {fp8_word(z[0], z[1], z[2], z[3]), fp8_word(z[4], z[5], z[6], z[7])};
            *reinterpret_cast<u32x2 *>(q) = w;
            if (bounds) {
              fp8_values(w[0], z);
              fp8_values(w[1], z + 4);
            }
          } else {
            const u32x4 w = {pack_act<ACT>(z[0], z[1]), pack_act<ACT>(z[2], z[3]),
                             pack_act<ACT>(z[4], z[5]), pack_act<ACT>(z[6], z[7])};
            *reinterpret_cast<u32x4 *>(q) = w;
            if (bounds) {
#pragma unroll
              for (int i = 0; i < 8; ++i)
                z[i] = act_to_float<ACT>((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
            }
          }
          if (bounds) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              lo[n * 8 + i] = fminf(lo[n * 8 + i], z[i]);
              hi[n * 8 + i] = fmaxf(hi[n * 8 + i], z[i]);
            }
          }
        }
      };
#pragma unroll
      for (int k = 0; k < KEEP; ++k)
        if (t0 + k * TW < m.n) store(t0 + k * TW, x[k], scales[k]);
      if constexpr (!ONE)
        for (int t = t0 + KEEP * TW; t < m.n; t += TW) {
          float y[16];
          const float by = fetch(t, plane, y);
          store(t, y, by);
        }
      if (bounds) {
        if constexpr (FP8) {  // of codes until here, all in units of the scale
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            lo[i] *= scale;
            hi[i] *= scale;
          }
        }
        write_bounds<LP>(kv, m.page, h, lane, at, lo, hi);
      }
    }
  }
}

template <int ACT, bool FP8, int LP>
void move_as(const MoveArgs &a, hipStream_t s) {
  const uint32_t units = (uint32_t)((a.layers + a.layers_wave - 1) / a.layers_wave * a.n_seqs *
                                    a.blocks_most);
  const dim3 grid((units + kWaves - 1) / kWaves), block(kThreads);
  const bool halves = !a.rope || (!a.interleaved && a.rope_dim % 16 == 0);
  if (!halves)
    hipLaunchKernelGGL((move_tokens<ACT, FP8, LP, false, false>), grid, block, 0, s, a, units);
  else if (a.kv.page_tokens <= 16)
    hipLaunchKernelGGL((move_tokens<ACT, FP8, LP, true, true>), grid, block, 0, s, a, units);
  else
    hipLaunchKernelGGL((move_tokens<ACT, FP8, LP, true, false>), grid, block, 0, s, a, units);
}

template <int ACT, bool FP8>
hipError_t move(const MoveArgs &a, hipStream_t s) {
  switch (lanes_of(a.kv.head_dim)) {
    case 4: move_as<ACT, FP8, 4>(a, s); break;
    case 8: move_as<ACT, FP8, 8>(a, s); break;
    default: move_as<ACT, FP8, 16>(a, s);
  }
  return hipGetLastError();
}

}  // namespace

int32_t copy_runs(int64_t piece) { return (int32_t)((piece + kRun - 1) / kRun); }

hipError_t launch_copy_pages(const CopyArgs &a, hipStream_t s) {
  (void)hipGetLastError();
  const int64_t runs = (int64_t)a.n * a.layers * a.runs_piece;
  bool planes = false;
  for (int k = 0; k < kCopyPlanes; ++k) planes = planes || a.plane[k];
  const int64_t units = runs + (planes ? (int64_t)a.n * a.layers : 0);
  hipLaunchKernelGGL(copy_pages, dim3((unsigned)((units + kWaves - 1) / kWaves)), dim3(kThreads),
                     0, s, a, runs, units);
  return hipGetLastError();
}

hipError_t launch_move_tokens(const MoveArgs &a, int act, int fp8, hipStream_t s) {
  (void)hipGetLastError();
  if (fp8) return move<kBf16, true>(a, s);
  return act == kBf16 ? move<kBf16, false>(a, s) : move<kF16, false>(a, s);
}

}  // namespace ea
