// Large batches: equal slices of the batch's steps, one per wavefront, whatever the
// lengths are.
//
// The line: each (request, kv head) pair with steps occupies kSlicePairCost positions,
// what a wavefront loses between two pairs, and one for every step. Wavefront s owns the
// positions of slice s. Its steps, whatever pairs they belong to, are one sequence: while
// a step is computed the next one's tiles are in flight, also across the end of a pair,
// and the next pair's query rows were requested a pair earlier. A pair that slices cut
// is merged from their shares by the last to finish.
//
// Where a workgroup's wavefronts hold several shares of a pair they are merged in LDS by
// the last of them, and only one share per workgroup and pair passes through the
// workspace.
//
// A workgroup of four (bf16) or eight (packed) wavefronts per compute unit, so that each
// holds two tiles of 8 KiB in registers without spilling; more wavefronts with one tile
// each, K and V apart, were slower. What a call pays besides its bytes is about 10 us: two
// reads of the lengths, the first tiles' latency, the merges.
#pragma once

#include "shaped.h"

namespace neo {
namespace {

constexpr int32_t kSlicePairCost = 1;
constexpr int32_t kSliceMinPositions = 2;  // no slice of less than a pair's cost and a step

template <class C>
__device__ inline float natural_lse(const ShapedParams& p, int32_t g, int h, const Seen& seen,
                                    float m, float l) {
  return (m + __log2f(l)) * kLn2 + left_out<C>(p, g, h, seen);
}

// Output row `row` (head h of kv head g) from k partials, the i-th in slot
// slot_of(i). Lane l owns dims 2l, 2l + 1.
template <class C, class SlotOf>
__device__ inline void merge_row(const ShapedParams& p, int32_t row, int32_t g, int h,
                                 const Seen& seen, int32_t k, SlotOf slot_of, int lane) {
  constexpr int G = C::G;
  constexpr int kBatch = 16;
  float m = kLowest, l = 0.f, x = 0.f, y = 0.f;
  for (int32_t base = 0; base < k; base += kWave) {
    const int32_t cnt = min(kWave, k - base);
    const size_t mine = slot_of(base + min(lane, cnt - 1));
    const float2 ml = load_coherent2(p.part_ml + (mine * G + h) * 2);
    float2 v[kBatch];
    auto load = [&](int32_t i0) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        v[u] = load_coherent2(
            p.part_o + ((size_t)slot_of(base + min(i0 + u, cnt - 1)) * G + h) * kHeadDim +
            2 * lane);
    };
    load(0);
    const float mc = fmaxf(m, wave_max_f32(ml.x));
    const float w = lane < cnt ? __builtin_amdgcn_exp2f(ml.x - mc) : 0.f;
    const float scale = __builtin_amdgcn_exp2f(m - mc);  // 0 on the first round
    m = mc;
    l = l * scale + wave_sum_f32(lane < cnt ? w * ml.y : 0.f);
    x *= scale;
    y *= scale;
    for (int32_t i0 = 0; i0 < cnt; i0 += kBatch) {
      if (i0 > 0) load(i0);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (i0 + u >= cnt) break;
        const float wi = __builtin_bit_cast(
            float, __builtin_amdgcn_readlane(__builtin_bit_cast(int32_t, w), i0 + u));
        x = fmaf(wi, v[u].x, x);
        y = fmaf(wi, v[u].y, y);
      }
    }
  }
  const float inv = 1.f / l;
  *reinterpret_cast<float2*>(p.out + (size_t)row * kHeadDim + 2 * lane) =
      float2{x * inv, y * inv};
  if (p.lse && lane == 0) p.lse[row] = natural_lse<C>(p, g, h, seen, m, l);
}

// All heads of a pair that slices cut, from k partials, the i-th in slot slot_of(i). The
// heads' reads do not wait for one another: a round trip for their maxima and the first
// rows together, and one for every few partials after those.
template <class C, class SlotOf>
__device__ inline void merge_pair_rows(const ShapedParams& p, int32_t b, int32_t g,
                                       const Seen& seen, int32_t k, SlotOf slot_of, int lane) {
  constexpr int G = C::G;
  constexpr int kHeads = G < 8 ? G : 8;
  constexpr int kBatch = 16 / kHeads;
  const int32_t row0 = b * p.hq + g * G;
  for (int h0 = 0; h0 < G; h0 += kHeads) {
    float m[kHeads], l[kHeads];
    float2 x[kHeads];
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      m[u] = kLowest;
      l[u] = 0.f;
      x[u] = float2{0.f, 0.f};
    }
    for (int32_t base = 0; base < k; base += kWave) {
      const int32_t cnt = min(kWave, k - base);
      float2 v[kBatch][kHeads], ml[kHeads];
      const size_t mine = slot_of(base + min(lane, cnt - 1));
#pragma unroll
      for (int u = 0; u < kHeads; ++u)
        ml[u] = load_coherent2(p.part_ml + (mine * G + h0 + u) * 2);
      auto load = [&](int32_t i0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const size_t slot = slot_of(base + min(i0 + i, cnt - 1));
#pragma unroll
          for (int u = 0; u < kHeads; ++u)
            v[i][u] = load_coherent2(p.part_o + (slot * G + h0 + u) * kHeadDim + 2 * lane);
        }
      };
      load(0);
      float w[kHeads];
#pragma unroll
      for (int u = 0; u < kHeads; ++u) {
        const float mc = fmaxf(m[u], wave_max_f32(ml[u].x));
        const float scale = __builtin_amdgcn_exp2f(m[u] - mc);  // 0 on the first round
        w[u] = lane < cnt ? __builtin_amdgcn_exp2f(ml[u].x - mc) : 0.f;
        l[u] = l[u] * scale + wave_sum_f32(lane < cnt ? w[u] * ml[u].y : 0.f);
        x[u].x *= scale;
        x[u].y *= scale;
        m[u] = mc;
      }
      for (int32_t i0 = 0; i0 < cnt; i0 += kBatch) {
        if (i0 > 0) load(i0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          if (i0 + i >= cnt) break;
#pragma unroll
          for (int u = 0; u < kHeads; ++u) {
            const float wi = __builtin_bit_cast(
                float, __builtin_amdgcn_readlane(__builtin_bit_cast(int32_t, w[u]), i0 + i));
            x[u].x = fmaf(wi, v[i][u].x, x[u].x);
            x[u].y = fmaf(wi, v[i][u].y, x[u].y);
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const float inv = 1.f / l[u];
      const int h = h0 + u;
      *reinterpret_cast<float2*>(p.out + (size_t)(row0 + h) * kHeadDim + 2 * lane) =
          float2{x[u].x * inv, x[u].y * inv};
      if (p.lse && lane == 0) p.lse[row0 + h] = natural_lse<C>(p, g, h, seen, m[u], l[u]);
    }
  }
}

template <class C>
__device__ inline int32_t steps_of(int32_t blocks) {
  return (blocks + C::kStep - 1) / C::kStep;
}
template <class C>
__device__ inline int32_t line_weight(int32_t blocks) {
  return blocks > 0 ? steps_of<C>(blocks) + kSlicePairCost : 0;
}

// The line as a wavefront sees it: its slice and the pair that holds its first position.
struct LineStart {
  SliceGeom geo;
  int32_t s0, s1;   // this wavefront's positions
  int32_t b, g, x;  // pair (request, kv head) and the offset of s0 in it
};

// Every thread sums a run of requests and the workgroup scans the sums; each wavefront
// finds the run that holds its first position and walks it. Any batch, two reads of the
// lengths. False where the wavefront has no slice.
template <class C>
__device__ inline bool find_slice(const ShapedParams& p, LineStart& at) {
  constexpr int kWaves = C::kSliceWaves;
  constexpr int kThreads = kWave * kWaves;
  __shared__ int32_t ends[kThreads];  // weights up to the end of each thread's run
  __shared__ int32_t waves[kWaves];
  const int lane = threadIdx.x & (kWave - 1);
  const int wv = uniform(threadIdx.x >> 6);
  const int32_t run = (p.batch - 1) / kThreads + 1;
  const int32_t b0 = min(p.batch, (int32_t)threadIdx.x * run), b1 = min(p.batch, b0 + run);
  int32_t sum = 0;
  for (int32_t b = b0; b < b1; ++b) sum += line_weight<C>(lane_seen(p, b).n);
  int32_t incl = wave_incl_scan_i32(sum);
  if (lane == kWave - 1) waves[wv] = incl;
  __syncthreads();
  int32_t W = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wv) incl += waves[w];
    W += waves[w];
  }
  ends[threadIdx.x] = incl;
  __syncthreads();
  W = uniform(W) * p.hkv;
  const int32_t n = min((int32_t)gridDim.x * kWaves, max(1, W / kSliceMinPositions));
  const int32_t slice = (int32_t)blockIdx.x * kWaves + wv;
  at.geo = make_uniform(make_slice_geom(W, n, false));
  if (W == 0 || slice >= n) return false;
  at.s0 = slice_start_u(slice, at.geo);
  at.s1 = slice_start_u(slice + 1, at.geo);
  // The first run that ends behind s0: kWaves runs a lane, ascending.
  int32_t passed = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i)
    passed += ends[lane * kWaves + i] * p.hkv <= at.s0 ? 1 : 0;
  const int32_t r = wave_sum_i32(passed);
  int32_t before = r > 0 ? uniform(ends[r - 1]) : 0, w = 1;
  int32_t b = r * run;
  for (;; ++b) {
    w = line_weight<C>(load_seen(p, b).n);
    if (at.s0 < (before + w) * p.hkv) break;
    before += w;
  }
  const int32_t rem = at.s0 - before * p.hkv;
  at.b = uniform(b);
  at.g = uniform(rem / w);
  at.x = uniform(rem % w);
  return at.s0 < at.s1;
}

// The share of a pair that a slice holds: steps [j0, jend) of the pair, whose steps
// start at position first; step j is the next.
struct Segment {
  Place at;
  int32_t first, j0, j, jend;
};

// Slots of rows in LDS, a set of them for every wavefront: slot 0 for its share of a pair
// that runs into its slice, slot 1 of one that starts in it, until the last wavefront of
// the workgroup that has a share of that pair merges them. The others collect finished
// rows: written as each is ready, their stores stand in the queue of the loads, and
// HBM turns between reading and writing for every few kilobytes. (With 16 heads there
// is no room for more, and slot 1 turns a pair's rows for writing; its share there, if it
// has one, is its last.)
template <class C>
struct SliceShared {
  static constexpr int kSets = 155 * 1024 / (C::kSliceWaves * C::G * kHeadDim * 4);
  static constexpr int kFinished = kSets - 2 > 8 ? 8 : (kSets > 2 ? kSets - 2 : 1);
  static constexpr int kFirstFinished = kSets > 2 ? 2 : 1;
  static constexpr int kSlots = kFirstFinished + kFinished;
  static_assert(kSets >= 2, "two slots for shares");
  float rows[C::kSliceWaves][kSlots][C::G * kHeadDim];  // word c of row h at c ^ h
  float2 ml[C::kSliceWaves][2][C::G];
  float lse[C::kSliceWaves][kFinished][C::G];
  int32_t row0[C::kSliceWaves][kFinished];  // first output row of each finished slot
  int32_t count[C::kSliceWaves][2];  // of the pair whose first share here is that one
};

template <class C>
__global__ __launch_bounds__(kWave* C::kSliceWaves, C::kSliceWaves / 4) void slice_kernel(
    ShapedParams p) {
  constexpr int G = C::G;
  constexpr int kWaves = C::kSliceWaves;
  __shared__ SliceShared<C> sh;
  const int lane = threadIdx.x & (kWave - 1);
  const int wv = uniform(threadIdx.x >> 6);
  if (threadIdx.x < 2 * kWaves) (&sh.count[0][0])[threadIdx.x] = 0;
  LineStart at;
  const bool any = find_slice<C>(p, at);  // (its barriers stand behind the counts' clearing)
  const int32_t first_slice = (int32_t)blockIdx.x * kWaves;
  const int32_t slice = first_slice + wv;
  // Requests that see nothing: a wavefront's share of them.
  for (int32_t b = slice; b < p.batch; b += (int32_t)gridDim.x * kWaves) {
    if (load_seen(p, b).n != 0) continue;
    for (int i = lane; i < p.hq * kHeadDim; i += kWave)
      p.out[(size_t)b * p.hq * kHeadDim + i] = 0.f;
    if (p.lse)
      for (int i = lane; i < p.hq; i += kWave) p.lse[(size_t)b * p.hq + i] = -INFINITY;
  }
  if (!any) return;
  const SliceGeom geo = at.geo;
  // Where slice c keeps its share of a pair whose steps start at `first`, and a workgroup
  // its wavefronts' shares together.
  auto which = [&](int32_t c, int32_t first) { return first <= slice_start(c, geo) ? 0 : 1; };
  auto group_slot = [&](int32_t wg, int32_t c0) { return 2 * wg + (c0 < wg * kWaves ? 0 : 1); };

  Segment cur, nxt;
  cur.at = Place{at.b, at.g, load_seen(p, at.b)};
  cur.first = at.s0 - at.x + kSlicePairCost;
  cur.j = cur.j0 = max(0, at.x - kSlicePairCost);
  cur.jend = min(steps_of<C>(cur.at.seen.n), at.s1 - cur.first);
  if (cur.jend <= cur.j) return;  // the slice ends before the pair's next step
  const int32_t s1 = at.s1;
  // The slice's next segment, from its pair's step 0 on. Where there is none its jend is 0
  // and its pair this one.
  auto find_next = [&]() {
    nxt = cur;
    nxt.j = nxt.j0 = nxt.jend = 0;
    const int32_t pos = cur.first + steps_of<C>(cur.at.seen.n);
    if (pos >= s1) return;
    int32_t b = cur.at.b, g = cur.at.g + 1;
    Seen seen = cur.at.seen;
    if (g == p.hkv) {
      g = 0;
      do {
        if (++b >= p.batch) return;
        seen = load_seen(p, b);
      } while (seen.n == 0);
    }
    nxt.first = pos + kSlicePairCost;
    nxt.jend = min(steps_of<C>(seen.n), s1 - nxt.first);
    if (nxt.jend <= 0)
      nxt.jend = 0;
    else
      nxt.at = Place{b, g, seen};
  };
  find_next();
  auto q_rows = [&](const Place& at) {
    return p.q + ((size_t)at.b * p.hq + at.g * G) * kHeadDim;
  };
  Pair<C> pr = make_pair<C>(p, cur.at, lane);
  typename C::Q qn;
  Softmax st;
  st.init();

  // A pair that this wavefront has to merge from workgroups' shares, once it has arrived
  // last. The first segment's share is counted a step after it is stored, when the stores
  // are complete, and the count looked at in the end.
  struct Cut {
    int32_t b, g, c0, wg0, k;
  } early{}, late{};
  bool early_due = false, early_cut = false, late_last = false;
  int32_t early_old = 0;
  auto count = [&](const Cut& c) {
    int32_t old = 0;
    if (lane == 0)
      old = __hip_atomic_fetch_add(p.counters + c.wg0, 1, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
    return old;
  };
  auto arrived_last = [&](const Cut& c, int32_t old) -> bool {
    if (__builtin_amdgcn_readlane(old, 0) != c.k - 1) return false;
    if (lane == 0)
      __hip_atomic_store(p.counters + c.wg0, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
  };

  // Finished rows, to be written later.
  using Shared = SliceShared<C>;
  int32_t finished = 0;
  auto flush = [&]() {
    wave_sync_lds();
    for (int s = 0; s < finished; ++s) {
      const float* slot = sh.rows[wv][Shared::kFirstFinished + s];
      const int32_t row0 = uniform(sh.row0[wv][s]);
      f32x4_t* out = reinterpret_cast<f32x4_t*>(p.out + (size_t)row0 * kHeadDim);
#pragma unroll
      for (int i = 0; i < (G * 32 + kWave - 1) / kWave; ++i) {
        const int w = i * kWave + lane;  // 16-byte word
        if (G * 32 % kWave == 0 || w < G * 32)
          __builtin_nontemporal_store(
              *reinterpret_cast<const f32x4_t*>(slot + 4 * (w ^ (w >> 5))), out + w);
      }
      if (p.lse && lane < G) p.lse[row0 + lane] = sh.lse[wv][s][lane];
    }
    wave_sync_lds();
    finished = 0;
  };
  auto next_finished = [&](int32_t row0) -> int {  // the slot's number
    if (finished == Shared::kFinished) flush();
    sh.row0[wv][finished] = row0;  // every lane: the same value
    return finished++;
  };
  auto to_slot = [&](int slot, float by) {
    const int h = lane & 15;
    if (h < G)
      C::each_word(st.acc, lane, [&](int c, f32x4_t v) {
        *reinterpret_cast<f32x4_t*>(&sh.rows[wv][slot][h * kHeadDim + 4 * (c ^ h)]) = v * by;
      });
  };
  auto finish = [&]() {
    C::fold(st.acc);
    const float l = C::head_sum(st.l);
    const int h = lane & 15;
    const int32_t row0 = cur.at.b * p.hq + cur.at.g * G;
    const int32_t steps = steps_of<C>(cur.at.seen.n);
    if (cur.j0 == 0 && cur.jend == steps) {
      const int s = next_finished(row0);
      to_slot(Shared::kFirstFinished + s, 1.f / l);
      if (lane < G) sh.lse[wv][s][h] = natural_lse<C>(p, cur.at.g, h, cur.at.seen, st.m, l);
      return;
    }
    const int mine = uniform(which(slice, cur.first));
    if (Shared::kFirstFinished == 1 && mine == 1) flush();  // (the slot turned rows so far)
    to_slot(mine, 1.f);
    if (lane < G) sh.ml[wv][mine][h] = float2{st.m, l};
    const int32_t c0 = uniform(slice_of(cur.first, geo));
    const int32_t c1 = uniform(slice_of(cur.first + steps - 1, geo));
    const int32_t w0 = max(c0, first_slice), w1 = min(c1, first_slice + kWaves - 1);
    // A wavefront's LDS operations complete in order: the count follows the rows.
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(kWaitLgkmcnt0);
    if (w0 < w1) {
      int32_t old = 0;
      if (lane == 0)
        old = __hip_atomic_fetch_add(&sh.count[w0 - first_slice][which(w0, cur.first)], 1,
                                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      old = __builtin_amdgcn_readlane(old, 0);
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      if (old != w1 - w0) return;
    }
    const int32_t wg = blockIdx.x;
    const bool complete = w0 == c0 && w1 == c1;
    const size_t slot = (size_t)group_slot(wg, c0);
    // With 16 heads a complete pair's rows are written at once: its slot may be in use.
    const bool keep = complete && Shared::kFirstFinished > 1;
    const int s = keep ? next_finished(row0) : 0;
    // Lane hh holds head hh's maximum and denominator; a row's reads do not wait for
    // those of the others.
    const int hl = lane & (G - 1);
    float m = kLowest, sum = 0.f;
    float2 row[G];
#pragma unroll
    for (int hh = 0; hh < G; ++hh) row[hh] = float2{0.f, 0.f};
    for (int32_t c = w0; c <= w1; ++c)
      m = fmaxf(m, sh.ml[c - first_slice][which(c, cur.first)][hl].x);
    for (int32_t c = w0; c <= w1; ++c) {
      const int w = c - first_slice, k = which(c, cur.first);
      const float2 ml = sh.ml[w][k][hl];
      const float e = __builtin_amdgcn_exp2f(ml.x - m);
      sum = fmaf(e, ml.y, sum);
      const float* rows = sh.rows[w][k];
#pragma unroll
      for (int hh = 0; hh < G; ++hh) {
        const float2 v =
            *reinterpret_cast<const float2*>(rows + hh * kHeadDim + ((2 * lane) ^ (4 * hh)));
        const float eh = __builtin_bit_cast(
            float, __builtin_amdgcn_readlane(__builtin_bit_cast(int32_t, e), hh));
        row[hh].x = fmaf(eh, v.x, row[hh].x);
        row[hh].y = fmaf(eh, v.y, row[hh].y);
      }
    }
    if (complete) {
      const float inv = 1.f / sum;
      const float lse = natural_lse<C>(p, cur.at.g, hl, cur.at.seen, m, sum);
      if (keep) {
        if (lane < G) sh.lse[wv][s][hl] = lse;
      } else {
        if (p.lse && lane < G) p.lse[row0 + hl] = lse;
      }
      float* rows = keep ? sh.rows[wv][Shared::kFirstFinished + s] : nullptr;
#pragma unroll
      for (int hh = 0; hh < G; ++hh) {
        const float ih = __builtin_bit_cast(
            float, __builtin_amdgcn_readlane(__builtin_bit_cast(int32_t, inv), hh));
        const float2 r{row[hh].x * ih, row[hh].y * ih};
        if (keep)
          *reinterpret_cast<float2*>(rows + hh * kHeadDim + ((2 * lane) ^ (4 * hh))) = r;
        else
          *reinterpret_cast<float2*>(p.out + (size_t)(row0 + hh) * kHeadDim + 2 * lane) = r;
      }
      return;
    }
#pragma unroll
    for (int hh = 0; hh < G; ++hh)
      store_coherent2(p.part_o + (slot * G + hh) * kHeadDim + 2 * lane, row[hh].x, row[hh].y);
    if (lane < G) store_coherent2(p.part_ml + (slot * G + hl) * 2, m, sum);
    const int32_t wg0 = c0 / kWaves;
    const Cut cut{cur.at.b, cur.at.g, c0, wg0, c1 / kWaves - wg0 + 1};
    if (nxt.jend > 0) {
      early = cut;
      early_due = early_cut = true;
    } else {
      late = cut;
      flush();
      wait_all_memory();
      late_last = arrived_last(cut, count(cut));
    }
  };

  // The block ids of the step after the next one, where it is known.
  Blocks<C> ids;
  bool known = false;
  // Of the step after step cur.j.
  auto next_blocks = [&]() {
    const bool more = cur.j + 1 < cur.jend;
    if (!known) ids = find_blocks<C>(p, more ? cur.at : nxt.at, more ? cur.j + 1 : 0);
    return ids;
  };
  auto find_ids = [&]() {
    const bool more = cur.j + 1 < cur.jend;
    known = more || nxt.jend > 1;
    if (!known) return;
    const bool in = cur.j + 2 < cur.jend;
    ids = find_blocks<C>(p, in ? cur.at : nxt.at, in ? cur.j + 2 : (more ? 0 : 1));
  };
  auto count_early = [&]() {
    if (!early_due) return;
    // The share was stored before the newest step's loads were issued.
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(C::kWaitOneStep);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    early_old = count(early);
    early_due = false;
  };
  // Step cur.j is in `t`; the tiles of the one after it are requested into `tn`, and the
  // next pair's query rows once more. (The wait counts are the compiler's: where two paths
  // join it assumes the one with fewer operations in flight. Rows requested where a
  // segment ends would be waited for at once; requested at every step, from the cache,
  // they are a step old when they are waited for.) False after the slice's last step.
  auto step = [&](typename C::Tile& t, typename C::Tile& tn) -> bool {
    const bool more = cur.j + 1 < cur.jend;
    load_step<C, true, true>(p, more ? cur.at : nxt.at, next_blocks(), tn, lane);
    C::load_q(qn, q_rows(nxt.at), lane);
    find_ids();
    count_early();
    attend_step<C>(p, cur.at.seen, pr, t, cur.j, st, lane);
    if (++cur.j < cur.jend) return true;
    finish();
    if (nxt.jend == 0) return false;
    cur = nxt;
    st.init();
    find_next();
    pr.q = qn;
    set_bias<C>(p, cur.at, pr, lane);
    return true;
  };
  typename C::Tile t0, t1;
  load_step<C, true, true>(p, cur.at, find_blocks<C>(p, cur.at, cur.j), t0, lane);
  while (step(t0, t1) && step(t1, t0)) {
  }
  flush();
  auto merge = [&](const Cut& c) {
    merge_pair_rows<C>(p, c.b, c.g, load_seen(p, c.b), c.k,
                       [&](int32_t i) { return (size_t)group_slot(c.wg0 + i, c.c0); }, lane);
  };
  if (late_last) merge(late);
  if (early_cut && arrived_last(early, early_old)) merge(early);
}

}  // namespace
}  // namespace neo
