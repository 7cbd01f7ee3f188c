// Eviction: of each (request, kv head), the newest tokens and those with the
// largest sums of attention weights are moved, in their order, to new blocks.
//
// Two kernels. The first finds which tokens stay, one workgroup per (request, kv
// head): the sums as integers of the same order, the k-th largest of them by four
// rounds of 256 counts (eight bits of it a round), then a running count in token
// order; equal sums stay from the lowest token on. The second moves the tokens'
// keys and values, one wavefront per new (block, kv head) tile. Source blocks are
// only read, so blocks that several requests share may be evicted from.
//
// One row's selection is a chain of four rounds, each a pass and two barriers; a workgroup
// per row leaves most of the chip idle for small batches, and other splits would pay the
// same barriers across workgroups. The move is bound by HBM's lines: a packed token is 136
// bytes in 34 pieces of a record, and of 16 tokens scattered over their blocks nearly every
// line is fetched whole (96 requests of 2048 to 8192 tokens to 1500: 124 us for 339 MB of
// tokens, about 690 MB of lines, 5.6 TB/s).
#include "decode_common.h"
#include "packed.h"
#include "shaped_ops.h"

namespace neo {
namespace {

constexpr int kSelectWaves = 16;
constexpr int kSelectThreads = kWave * kSelectWaves;
constexpr int kBins = 256;
// Requests whose table allows up to this many tokens have their sums read once and kept in
// LDS: 10.7 us for one request of 8 heads and 4099 tokens, where six passes over L2 take
// 11.1, and 33 us against 37 for 96 requests of 2048 to 8192 tokens. (Counting 12 bits at
// first and ranking the rest directly: 12.2 and 39; in registers, unrolled: 17.5 and 35.)
constexpr int32_t kOnceTokens = 8192;

// Unsigned integers in the order of the sums; both zeros are the same, and a NaN
// counts as the largest, so that what is not understood stays.
__device__ inline uint32_t order_of(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  if ((u << 1) == 0) return 0x80000000u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <bool kOnce>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictParams p) {
  __shared__ float once[kOnce ? kOnceTokens : 1];
  __shared__ int32_t bins[kBins];
  __shared__ int32_t state[2];  // the bin that holds the k-th largest, what is left of k there
  __shared__ int32_t above[kSelectWaves], equal[kSelectWaves];
  const int lane = threadIdx.x & (kWave - 1);
  const int wv = uniform(threadIdx.x >> 6);
  const int32_t b = blockIdx.x / p.hkv, g = blockIdx.x % p.hkv;
  const int32_t L = uniform(clamp_len(p.lens[b], p.mbps));
  const int32_t n = uniform(min(L, min(max(p.budgets[b], 0), p.new_mbps * kBlock)));
  const int32_t old = L - min(max(p.recent, 0), n);  // tokens that compete
  const int32_t k = n - (L - old);                   // and how many of them stay
  const int32_t slots = p.new_mbps * kBlock;
  const float* sums = p.sums + ((size_t)b * p.hkv + g) * (size_t)p.sums_stride;
  int32_t* kept = p.kept + ((size_t)b * p.hkv + g) * (size_t)slots;
  float* new_sums = p.new_sums + ((size_t)b * p.hkv + g) * (size_t)slots;
  auto sum_of = [&](int32_t t) { return kOnce ? once[t] : sums[t]; };
  if constexpr (kOnce) {
#pragma unroll 4
    for (int32_t t = threadIdx.x; t < old; t += kSelectThreads) once[t] = sums[t];
    __syncthreads();
  }
  if (g == 0 && threadIdx.x == 0) p.new_lens[b] = n;
  for (int32_t i = n + threadIdx.x; i < slots; i += kSelectThreads) {
    kept[i] = -1;
    new_sums[i] = 0.f;
  }
  // The k-th largest, from its highest byte down: `prefix` are the bytes found.
  uint32_t prefix = 0;
  int32_t left = k;
  const bool all = k == old, none = k == 0;
  if (!all && !none) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < kBins; i += kSelectThreads) bins[i] = 0;
      __syncthreads();
      for (int32_t t = threadIdx.x; t < old; t += kSelectThreads) {
        const uint32_t u = order_of(sum_of(t));
        if (shift == 24 || (u >> (shift + 8)) == prefix)
          atomicAdd(&bins[(u >> shift) & 0xFF], 1);
      }
      __syncthreads();
      if (wv == 0) {  // lane l: bins 255 - 4l .. 252 - 4l, from the largest on
        int32_t c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += c[i] = bins[kBins - 1 - (4 * lane + i)];
        int32_t before = wave_incl_scan_i32(sum) - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < left && left <= before + c[i]) {
            state[0] = kBins - 1 - (4 * lane + i);
            state[1] = left - before;
          }
          before += c[i];
        }
      }
      __syncthreads();
      prefix = (prefix << 8) | (uint32_t)state[0];
      left = state[1];
    }
  }
  // Stays: a token above the k-th largest, the first `left` equal to it, and the
  // newest. Each wavefront counts its run of tokens, then places it.
  auto above_it = [&](uint32_t u) { return all || (!none && u > prefix); };
  auto equal_it = [&](uint32_t u) { return !all && !none && u == prefix; };
  const int32_t run = ((old - 1) / (kWave * kSelectWaves) + 1) * kWave;  // tokens of a wavefront
  const int32_t first = min(old, wv * run), last = min(old, first + run);
  int32_t ca = 0, ce = 0;
  for (int32_t t0 = first; t0 < last; t0 += kWave) {
    const int32_t t = t0 + lane;
    const uint32_t u = t < last ? order_of(sum_of(t)) : 0;
    ca += __popcll(__ballot(t < last && above_it(u)));
    ce += __popcll(__ballot(t < last && equal_it(u)));
  }
  if (lane == 0) {
    above[wv] = ca;
    equal[wv] = ce;
  }
  __syncthreads();
  int32_t at = 0, seen_equal = 0;  // tokens kept, and equal ones met, before this wavefront's
  for (int w = 0; w < wv; ++w) {
    at += above[w] + min(equal[w], max(0, left - seen_equal));
    seen_equal += equal[w];
  }
  const uint64_t below = (1ull << lane) - 1;
  for (int32_t t0 = first; t0 < last; t0 += kWave) {
    const int32_t t = t0 + lane;
    const float x = t < last ? sum_of(t) : 0.f;
    const uint32_t u = order_of(x);
    const uint64_t eq = __ballot(t < last && equal_it(u));
    const bool stays = t < last && (above_it(u) || (equal_it(u) && seen_equal + __popcll(eq & below) < left));
    const uint64_t st = __ballot(stays);
    if (stays) {
      const int32_t i = at + __popcll(st & below);
      kept[i] = t;
      new_sums[i] = x;
    }
    at += __popcll(st);
    seen_equal += __popcll(eq);
  }
  for (int32_t t = old + threadIdx.x; t < L; t += kSelectThreads) {
    kept[k + t - old] = t;
    new_sums[k + t - old] = sums[t];
  }
}

// One wavefront per (request, new block, kv head). Slots past the new length are
// set to zero.
constexpr int kMoveWaves = 4;
template <bool kPacked>
__global__ __launch_bounds__(kWave* kMoveWaves) void move_kernel(EvictParams p) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t tile = (int64_t)blockIdx.x * kMoveWaves + uniform(threadIdx.x >> 6);
  const int32_t g = (int32_t)(tile % p.hkv);
  const int64_t rest = tile / p.hkv;
  const int32_t j = (int32_t)(rest % p.new_mbps);
  const int64_t b64 = rest / p.new_mbps;
  if (b64 >= p.batch) return;
  const int32_t b = (int32_t)b64;
  // Lane l holds the place of token l % 16 of the new block, -1 behind the new length.
  const int32_t src =
      p.kept[((size_t)b * p.hkv + g) * (size_t)(p.new_mbps * kBlock) + j * kBlock + (lane & 15)];
  const int32_t dst_blk = p.new_table[(size_t)b * p.new_mbps + j];
  const bool real = src >= 0;
  const int count = __popcll(__ballot(real)) / 4;  // tokens of the block, the first ones
  if (count == 0 || dst_blk < 0 || dst_blk >= p.num_blocks) return;
  const int32_t sblk = p.table[(size_t)b * p.mbps + max(src, 0) / kBlock];
  const int64_t from = (int64_t)min((uint32_t)sblk, (uint32_t)(p.num_blocks - 1)) * p.blk_bytes +
                       (int64_t)g * (kPacked ? kPackedRecord : kTileBytes);
  const int sslot = src & (kBlock - 1);
  uint8_t* to = p.k + (int64_t)dst_blk * p.blk_bytes + (int64_t)g * (kPacked ? kPackedRecord : kTileBytes);
  auto from_of = [&](int slot) -> int64_t {
    const int32_t lo = __shfl((int32_t)(uint32_t)from, slot), hi = __shfl((int32_t)(from >> 32), slot);
    return (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
  };
  const u32x4_t zero = {0u, 0u, 0u, 0u};
  if constexpr (kPacked) {
    // As the lanes of a record: K of token l % 16, V of tokens 4 (l / 16) .. + 3.
    const int grp = lane >> 4, r = lane & 15;
    const uint8_t* rec = p.k + from;
    u32x4_t k = zero, v = zero;
    uint32_t ke = 0, ve = 0;
    if (real) {
      k = *reinterpret_cast<const u32x4_t*>(rec + grp * 256 + sslot * 16);
      ke = rec[packed_k_exp_at(sslot, grp)];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = 4 * grp + i;
      const uint8_t* vrec = p.k + from_of(slot);
      const int ss = __shfl(sslot, slot);
      if (slot < count) {
        v[i] = *reinterpret_cast<const uint32_t*>(vrec + packed_v_at(ss, r));
        if (r < 4) ve |= (uint32_t)vrec[packed_v_exp_at(ss, r)] << (8 * i);
      }
    }
    *reinterpret_cast<u32x4_t*>(to + 16 * lane) = k;
    *reinterpret_cast<u32x4_t*>(to + kPackedV + 16 * lane) = v;
    to[kPackedKExp + lane] = (uint8_t)ke;
    if (r < 4) *reinterpret_cast<uint32_t*>(to + kPackedVExp + 16 * grp + 4 * r) = ve;
  } else {
    // K: 16-byte pieces, four per lane; V: two dims per lane, token by token.
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int piece = 4 * i + (lane >> 4);
      u32x4_t w = zero;
      if (real) w = *reinterpret_cast<const u32x4_t*>(p.k + from + (piece * kBlock + sslot) * 16);
      *reinterpret_cast<u32x4_t*>(to + (piece * kBlock + (lane & 15)) * 16) = w;
    }
    uint8_t* vto = p.v + (to - p.k);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int d = 64 * half + lane;
      uint32_t w[8];
#pragma unroll
      for (int slot = 0; slot < kBlock; ++slot) {
        const uint8_t* vrec = p.v + from_of(slot);
        const int ss = __shfl(sslot, slot);
        uint32_t x = *reinterpret_cast<const uint16_t*>(vrec + (d * kBlock + ss) * 2);
        if (slot >= count) x = 0;
        w[slot / 2] = slot % 2 ? w[slot / 2] | (x << 16) : x;
      }
      u32x4_t* dst = reinterpret_cast<u32x4_t*>(vto + d * kBlock * 2);
      dst[0] = u32x4_t{w[0], w[1], w[2], w[3]};
      dst[1] = u32x4_t{w[4], w[5], w[6], w[7]};
    }
  }
}

}  // namespace

hipError_t launch_evict(const EvictParams& p, bool packed, hipStream_t stream) {
  if ((int64_t)p.mbps * kBlock <= kOnceTokens)
    select_kernel<true><<<(unsigned)(p.batch * p.hkv), kSelectThreads, 0, stream>>>(p);
  else
    select_kernel<false><<<(unsigned)(p.batch * p.hkv), kSelectThreads, 0, stream>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t tiles = (int64_t)p.batch * p.new_mbps * p.hkv;
  const unsigned grid = (unsigned)((tiles + kMoveWaves - 1) / kMoveWaves);
  if (packed)
    move_kernel<true><<<grid, kWave * kMoveWaves, 0, stream>>>(p);
  else
    move_kernel<false><<<grid, kWave * kMoveWaves, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace neo
