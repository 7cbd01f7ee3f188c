// Kernels of attention with shaped scores, and of the sums of its weights, over either
// cache type. Attention of few pairs: a workgroup of eight wavefronts takes a (request,
// kv head) pair or one of several equal shares of it. Such calls are short, and most of
// their time is latency: lengths, block ids, the first tiles, the merge in LDS and, between
// workgroups, through the workspace (one request of 877 tokens, 32/8 heads 8.9 us; packed, of
// 50021 tokens 18 us, where the loads alone take 16).
#pragma once

#include "shaped.h"
#include "shaped_slices.h"

namespace neo {
namespace {

constexpr int kShapedWaves = 8;
constexpr int kShapedThreads = kWave * kShapedWaves;
// A share has at least this many steps for every wavefront.
constexpr int32_t kStepsPerWave = 2;

// A workgroup's share of a pair, the s-th of n, and what the request sees.
struct Share {
  int32_t b, g, s, n;
  Seen seen;
};
// A pair has as many shares as `parts` and its steps allow; where it is so much longer than
// the others that a share would be more than two compute units' part of the whole call, it
// has more, and `spare` workgroups are there for those. (32 requests of 8 pairs, all of 512
// tokens but one of 100000: 92 us, 891 with `parts` alone; packed 38 and 380.) All wavefronts find the same; false where nothing
// is left for the workgroup.
template <class C>
__device__ inline bool find_share(const ShapedParams& p, int lane, Share& r) {
  auto seen_by = [&](int32_t b) {
    return b < p.batch ? lane_seen(p, b) : Seen{0, 0, 0, 0, 0, 0};
  };
  const Seen first = seen_by(lane);
  int32_t total = steps_of<C>(first.n);
  for (int32_t b = kWave + lane; b < p.batch; b += kWave) total += steps_of<C>(seen_by(b).n);
  total = uniform(wave_sum_i32(total)) * p.hkv;
  const int32_t limit = max(kShapedWaves * kStepsPerWave, total / p.spare + 1);
  const int32_t wg = (int32_t)blockIdx.x;
  int32_t before = 0;  // workgroups of the requests before
  for (int32_t b0 = 0; b0 < p.batch; b0 += kWave) {
    const Seen seen = b0 == 0 ? first : seen_by(b0 + lane);
    const int32_t steps = steps_of<C>(seen.n);
    const int32_t most = min(p.parts, (steps - 1) / (kShapedWaves * kStepsPerWave) + 1);
    const int32_t n = b0 + lane < p.batch ? max(1, max(most, (steps - 1) / limit + 1)) : 0;
    const int32_t incl = wave_incl_scan_i32(n);
    const uint64_t behind = __ballot((before + incl) * p.hkv > wg);
    if (behind) {
      const int f = __builtin_ctzll(behind);
      auto of = [&](int32_t v) { return __builtin_amdgcn_readlane(v, f); };
      r.n = of(n);
      const int32_t rem = wg - (before + of(incl) - r.n) * p.hkv;
      r.b = b0 + f;
      r.g = rem / r.n;
      r.s = rem % r.n;
      r.seen = Seen{of(seen.L), of(seen.p), of(seen.s), of(seen.pb), of(seen.f), of(seen.n)};
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, kWave - 1);
  }
  return false;
}

template <class C>
__global__ __launch_bounds__(kShapedThreads, 1) void attend_kernel(ShapedParams p) {
  constexpr int G = C::G;
  __shared__ float rows[kShapedWaves][G * kHeadDim];  // word c of row h at c ^ h
  __shared__ float ms[kShapedWaves][G], ls[kShapedWaves][G];
  __shared__ int32_t arrived;
  const int lane = threadIdx.x & (kWave - 1);
  const int wv = uniform(threadIdx.x >> 6);
  Share at;
  if (!find_share<C>(p, lane, at)) return;
  const Seen& seen = at.seen;
  const int32_t row0 = at.b * p.hq + at.g * G;
  float* out = p.out + (size_t)row0 * kHeadDim;
  if (seen.n == 0) {
    for (int i = threadIdx.x; i < G * kHeadDim; i += kShapedThreads) out[i] = 0.f;
    if (p.lse && threadIdx.x < G) p.lse[row0 + threadIdx.x] = -INFINITY;
    return;
  }
  const int32_t steps = steps_of<C>(seen.n), shares = at.n;
  const int32_t j0 = (int32_t)((int64_t)steps * at.s / shares);
  const int32_t j1 = (int32_t)((int64_t)steps * (at.s + 1) / shares);
  const int waves = min(kShapedWaves, j1 - j0);  // with steps, the first ones

  const Place place{at.b, at.g, seen};
  const Pair<C> pr = make_pair<C>(p, place, lane);
  Softmax st;
  st.init();
  each_step<C, typename C::Tile>(
      p, place, j0 + wv, j1, kShapedWaves,
      [&](typename C::Tile& t, const Blocks<C>& ids, int32_t) {
        load_step<C, true, true>(p, place, ids, t, lane);
      },
      [&](typename C::Tile& t, int32_t j) { attend_step<C>(p, seen, pr, t, j, st, lane); });
  if (wv < waves) {
    C::fold(st.acc);
    const float l = C::head_sum(st.l);
    const int h = lane & 15;
    if (h < G) {
      C::each_word(st.acc, lane, [&](int c, f32x4_t v) {
        *reinterpret_cast<f32x4_t*>(&rows[wv][h * kHeadDim + 4 * (c ^ h)]) = v;
      });
      if (lane < 16) {
        ms[wv][h] = st.m;
        ls[wv][h] = l;
      }
    }
  }
  __syncthreads();
  const int32_t pair = at.b * p.hkv + at.g;
  const size_t slot = blockIdx.x;
  for (int h = wv; h < G; h += kShapedWaves) {
    float m = kLowest, l = 0.f, x = 0.f, y = 0.f;
    for (int w = 0; w < waves; ++w) m = fmaxf(m, ms[w][h]);
    for (int w = 0; w < waves; ++w) {
      const float e = __builtin_amdgcn_exp2f(ms[w][h] - m);
      const float2 v =
          *reinterpret_cast<const float2*>(&rows[w][h * kHeadDim + ((2 * lane) ^ (4 * h))]);
      l = fmaf(e, ls[w][h], l);
      x = fmaf(e, v.x, x);
      y = fmaf(e, v.y, y);
    }
    if (shares == 1) {
      const float inv = 1.f / l;
      *reinterpret_cast<float2*>(out + h * kHeadDim + 2 * lane) = float2{x * inv, y * inv};
      if (p.lse && lane == 0) p.lse[row0 + h] = natural_lse<C>(p, at.g, h, seen, m, l);
    } else {
      store_coherent2(p.part_o + (slot * G + h) * kHeadDim + 2 * lane, x, y);
      if (lane == 0) store_coherent2(p.part_ml + (slot * G + h) * 2, m, l);
    }
  }
  if (shares == 1) return;
  // Every wavefront's stores are complete before the workgroup is counted; the
  // last workgroup of the pair merges it and leaves the counter at zero.
  wait_all_memory();
  __syncthreads();
  if (threadIdx.x == 0) {
    const int32_t old =
        __hip_atomic_fetch_add(p.counters + pair, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (old == shares - 1)
      __hip_atomic_store(p.counters + pair, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    arrived = old;
  }
  __syncthreads();
  if (arrived != shares - 1) return;
  const size_t slot0 = slot - at.s;
  for (int h = wv; h < G; h += kShapedWaves)
    merge_row<C>(p, row0 + h, at.g, h, seen, shares, [&](int32_t i) { return slot0 + i; }, lane);
}

// Sum over the heads of a token's weights: lanes of the 16-lane row (or of each
// half of it, where the columns hold the heads twice).
template <int kCtrl>
__device__ inline float dpp_f32(float v) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xF, 0xF, true));
}
template <bool kHalves>
__device__ inline float sum_over_columns(float v) {
  constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141;
  v += dpp_f32<kXor1>(v);
  v += dpp_f32<kXor2>(v);
  v += dpp_f32<kHalfMirror>(v);
  if constexpr (!kHalves) v += from_xor8(v);
  return v;
}

// The weights of steps [j0, j1) of a pair, added to their sums.
template <class C>
__device__ inline void add_weights(const ShapedParams& p, const Place& at, int32_t j0, int32_t j1,
                                   int lane) {
  const Seen& seen = at.seen;
  const Pair<C> pr = make_pair<C>(p, at, lane);
  const int h = C::head(lane), col = lane & 15;
  const bool real = h < C::G;
  // lse in base 2, without the bias of the pair's origin; one rounding, since
  // both may be large and nearly the same.
  float lse = 0.f;
  if (real) {
    const float slope = p.slopes ? p.slopes[at.g * C::G + h] : 0.f;
    const float d = slope < 0.f ? (float)(seen.first() - (seen.L - 1)) : 0.f;
    lse = fmaf(-slope, d, p.lse_in[at.b * p.hq + at.g * C::G + h]) * 1.4426950408889634f;
  }
  const size_t row = ((size_t)at.b * p.hkv + at.g) * (size_t)p.sums_stride;
  // A step's sums are requested with its keys: read when they are needed, they would be
  // waited for behind the next step's keys. Columns 0-3 (and 8-11) hold a token each.
  constexpr bool kHalves = C::kValues == 8;
  constexpr int kGroups = C::kValues / 4;
  struct Tile {
    typename C::Tile k;
    float sums[kGroups];
  };
  const int i = col & 3;
  const bool writes = kHalves ? (col & 4) == 0 : col < 4;
  const float* in = p.sums + row;
  float* out = p.sums_out + row;
  each_step<C, Tile>(
      p, at, j0, j1, 1,
      [&](Tile& t, const Blocks<C>& ids, int32_t j) {
        load_step<C, true, false>(p, at, ids, t.k, lane);
        int32_t first[C::kStep];
        first_tokens<C>(seen, j, first);
#pragma unroll
        for (int v = 0; v < kGroups; ++v)
          t.sums[v] = in[min(C::position(v, first, lane) + i, seen.L - 1)];
      },
      [&](Tile& t, int32_t j) {
        float x[C::kValues];
        const bool all = seen.sees_all(j * C::kStep, C::kStep);
        int32_t first[C::kStep];
        first_tokens<C>(seen, j, first);
        C::scores(t.k, pr.q, x, lane);
        const float factor = shape_scores<C>(p, seen, pr, first, all, x, lane);
#pragma unroll
        for (int v = 0; v < kGroups; ++v) {
          float w[4];
#pragma unroll
          for (int u = 0; u < 4; ++u)
            w[u] = sum_over_columns<kHalves>(
                real ? __builtin_amdgcn_exp2f(fmaf(x[4 * v + u], factor, -lse)) : 0.f);
          const float mine = i < 2 ? (i == 0 ? w[0] : w[1]) : (i == 2 ? w[2] : w[3]);
          const int32_t at_t = C::position(v, first, lane) + i;
          if (writes && seen.sees(at_t)) out[at_t] = t.sums[v] + mine;
        }
      });
}

// sums_out[b][g][t] = sums[b][g][t] + sum over the group's heads of exp(x_t - lse),
// for the tokens that the request sees. Reads K alone. Equal slices of the batch's steps,
// one per wavefront, as of attention over large batches; tokens need no merging. 64 requests
// of U[512, 2048] tokens, 32/8 heads: 32.5 us, 5.8 TB/s of keys and sums. Packed, 256 of
// U[256, 4096], 64/8 heads, capped: 68 us, 4.9 TB/s, or 5.2 with the whole lines of which the
// keys' exponents take half; the conversions and the caps are what is left beside the loads.
// (A workgroup per pair: 77.)
template <class C>
__global__ __launch_bounds__(kWave* C::kSliceWaves) void weights_kernel(ShapedParams p) {
  const int lane = threadIdx.x & (kWave - 1);
  LineStart at;
  if (!find_slice<C>(p, at)) return;
  Place pl{at.b, at.g, load_seen(p, at.b)};
  for (int32_t first = at.s0 - at.x + kSlicePairCost;;) {
    const int32_t steps = steps_of<C>(pl.seen.n);
    add_weights<C>(p, pl, max(0, at.s0 - first), min(steps, at.s1 - first), lane);
    first += steps;  // the next pair's position
    if (first >= at.s1) return;
    first += kSlicePairCost;
    if (++pl.g == p.hkv) {
      pl.g = 0;
      do {
        if (++pl.b >= p.batch) return;
        pl.seen = load_seen(p, pl.b);
      } while (pl.seen.n == 0);
    }
  }
}

}  // namespace

template <template <int> class Cache, int G>
hipError_t launch_shaped_g(const ShapedParams& p, bool weights, hipStream_t stream) {
  if (p.slices > 0 && !weights) {
    slice_kernel<Cache<G>><<<p.slices, kWave * Cache<G>::kSliceWaves, 0, stream>>>(p);
    return hipGetLastError();
  }
  if (weights)
    weights_kernel<Cache<G>><<<p.slices, kWave * Cache<G>::kSliceWaves, 0, stream>>>(p);
  else
    attend_kernel<Cache<G>>
        <<<p.batch * p.hkv * p.parts + p.spare, kShapedThreads, 0, stream>>>(p);
  return hipGetLastError();
}

template <template <int> class Cache>
hipError_t launch_shaped(const ShapedParams& p, int32_t group, bool weights, hipStream_t stream) {
  switch (group) {
    case 1: return launch_shaped_g<Cache, 1>(p, weights, stream);
    case 2: return launch_shaped_g<Cache, 2>(p, weights, stream);
    case 4: return launch_shaped_g<Cache, 4>(p, weights, stream);
    case 8: return launch_shaped_g<Cache, 8>(p, weights, stream);
    case 16: return launch_shaped_g<Cache, 16>(p, weights, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace neo
