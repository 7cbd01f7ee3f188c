// Decode attention with shaped scores: what the kernels over bf16 and packed
// caches share. For request b, L = lens[b], query head h and a token t that it
// sees (t < prefix[b] or t >= starts[b], below L):
//
//   x_t = scale * q_h . k_t;   x_t = cap * tanh(x_t / cap);   x_t += slope_h * (t - (L - 1))
//   out_h = sum_t exp(x_t - max x) v_t / sum_t exp(x_t - max x),   lse_h = log sum_t exp(x_t)
//
// Blocks without a token that is seen are neither read nor counted as work.
//
// One pass over a pair's tokens with the running maximum and sum of a softmax, products
// of 16 columns (the group's heads) on the matrix cores, sums in fp32. Over bf16 caches HBM
// bounds it (512 bytes a token and kv head; 256 requests of 64/8 heads that see 1500
// tokens, capped: 203 us, 6.6 TB/s). Over packed ones, with 136 bytes, the conversions,
// the products and the softmax of a wavefront no longer hide wholly behind the loads
// (512 requests of U[256, 4096] tokens: 223 us, 5.5 TB/s; the same loads without
// arithmetic 205), so what counts there is few instructions a token.
#pragma once

#include "decode_common.h"
#include "packed.h"

namespace neo {

struct ShapedParams {
  const uint16_t* q;        // [batch][hq][128] bf16
  const uint8_t* k;         // K of the bf16 cache, or the packed cache
  const uint8_t* v;         // V of the bf16 cache
  int64_t blk_bytes;        // bytes from one block to the next
  const int32_t* table;     // [batch][mbps]
  const int32_t* lens;      // [batch]
  const int32_t* starts;    // [batch] or null: 0
  const int32_t* prefix;    // [batch] or null: 0
  const float* slopes;      // [hq] or null: 0
  float* out;               // [batch][hq][128]
  float* lse;               // [batch][hq] or null
  float* part_o;            // partial rows, a slot of [group][128] each
  float* part_ml;           // their maxima and denominators, [group][2]
  int32_t* counters;        // arrivals, zero between calls
  const float* sums;        // weight sums [batch][hkv][sums_stride], read
  float* sums_out;          // and written
  const float* lse_in;      // [batch][hq]
  int64_t sums_stride;
  int32_t batch, hq, hkv, mbps, num_blocks;
  int32_t parts;            // workgroups of a (request, kv head) pair of usual length
  int32_t spare;            // and of all the longer ones together, more than that
  int32_t slices;           // workgroups of a call in slices, 0: in pairs
  float scale_log2;         // scale * log2(e)
  float cap_in, cap_log2;   // scale / cap and cap * log2(e); cap_log2 0: no cap
};

// What a request sees: tokens [0, p) and [s, L), in n blocks: the first pb, and
// those from block f on. Virtual block j is block_of(j) of the table row.
struct Seen {
  int32_t L, p, s, pb, f, n;
  __device__ int32_t block_of(int32_t j) const { return j < pb ? j : j - pb + f; }
  __device__ bool sees(int32_t t) const { return t < L && (t < p || t >= s); }
  __device__ int32_t first() const { return p > 0 ? 0 : s; }
  // Whether all tokens of the k virtual blocks from j on are seen.
  __device__ bool sees_all(int32_t j, int32_t k) const {
    return (j + k) * kBlock <= p ||
           (j >= pb && (j - pb + f) * kBlock >= s && (j + k - pb + f) * kBlock <= L);
  }
};
__device__ inline Seen make_seen(int32_t len, int32_t start, int32_t prefix, int32_t mbps) {
  Seen v;
  v.L = clamp_len(len, mbps);
  v.p = min(max(prefix, 0), v.L);
  v.s = min(max(start, v.p), v.L);
  if (v.s == v.p) v.s = v.p = 0;  // one range
  v.pb = (v.p + kBlock - 1) / kBlock;
  const int32_t nb = (v.L + kBlock - 1) / kBlock;
  v.f = v.s < v.L ? max(v.s / kBlock, v.pb) : nb;
  v.n = v.pb + nb - v.f;
  return v;
}

// Wave-uniform reads of the block table through the scalar cache: they neither
// occupy vector registers nor stand in the queue of the tile loads, whose
// in-order wait counts they would lengthen.
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;
__device__ inline ScalarInts scalar_ints(const int32_t* p) { return (ScalarInts)(uintptr_t)p; }

// Of a request that all lanes agree on.
__device__ inline Seen load_seen(const ShapedParams& p, int32_t b) {
  return make_seen(scalar_ints(p.lens)[b], p.starts ? scalar_ints(p.starts)[b] : 0,
                   p.prefix ? scalar_ints(p.prefix)[b] : 0, p.mbps);
}
// Of a request of each lane's own.
__device__ inline Seen lane_seen(const ShapedParams& p, int32_t b) {
  return make_seen(p.lens[b], p.starts ? p.starts[b] : 0, p.prefix ? p.prefix[b] : 0, p.mbps);
}

// A tile's words, from an address that all lanes agree on and an offset of each lane's.
// Every word is read once: nontemporal loads keep it from displacing what is used again.
template <class T>
__device__ inline T stream_load(const uint8_t* base, uint32_t off) {
  return __builtin_nontemporal_load(reinterpret_cast<const T*>(base + off));
}

// Lane l's value from lane l ^ 8 (a rotation of each 16-lane row by eight).
constexpr int kDppRowRor8 = 0x128;
__device__ inline uint32_t from_xor8(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppRowRor8, 0xF, 0xF, true);
}
__device__ inline float from_xor8(float v) {
  return __builtin_bit_cast(float, from_xor8(__builtin_bit_cast(uint32_t, v)));
}
// `other` of lane l ^ 8 in the upper (lower) eight lanes of each row, `own` in the rest.
__device__ inline uint32_t upper_from_xor8(uint32_t own, uint32_t other) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)own, (int)other, kDppRowRor8, 0xF, 0xC, false);
}
__device__ inline uint32_t lower_from_xor8(uint32_t own, uint32_t other) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)own, (int)other, kDppRowRor8, 0xF, 0x3, false);
}

// tanh to fp32 accuracy in the absolute sense that scores need: odd Taylor
// polynomial below kSmallTanh (the first term left out is 1e-8 of the value there),
// from the exponential above, where 1 - 2 / (e^2y + 1) cancels little.
constexpr float kSmallTanh = 0.3f;
__device__ inline float small_tanh(float y) {
  const float y2 = y * y;
  float r = fmaf(y2, -1382.f / 155925.f, 62.f / 2835.f);
  r = fmaf(y2, r, -17.f / 315.f);
  r = fmaf(y2, r, 2.f / 15.f);
  r = fmaf(y2, r, -1.f / 3.f);
  return fmaf(y * y2, r, y);
}
__device__ inline float any_tanh(float y) {
  const float e = __builtin_amdgcn_exp2f(fabsf(y) * 2.8853900817779268f);  // e^(2|y|)
  const float big = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f), y);
  return fabsf(y) < kSmallTanh ? small_tanh(y) : big;
}

// Four weights as sums of three bf16 numbers each, the leading eight of their 24 bits, the
// next and the last, so that nothing of them is lost; two to a register. (With two parts,
// 16 bits, a result is off by 1 to 2.5e-6 of itself, with three by the fp32 sums'
// roundings.)
__device__ inline void split_weights(const float* w, uint32_t (&parts)[3][2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float a = w[2 * i], b = w[2 * i + 1];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const uint32_t ua = __builtin_bit_cast(uint32_t, a), ub = __builtin_bit_cast(uint32_t, b);
      parts[k][i] = __builtin_amdgcn_perm(ub, ua, 0x07060302);
      a -= __builtin_bit_cast(float, ua & 0xFFFF0000u);
      b -= __builtin_bit_cast(float, ub & 0xFFFF0000u);
    }
  }
}

// ------------------------------------------------------------------ caches

// A cache type provides the matrix products over a step of kStep blocks. Each
// lane holds kValues scores of one head; position() tells which tokens they are.
//
// bf16: one block a step, the layouts and products of the plain decode kernel.
template <int G_>
struct Bf16Cache {
  static constexpr int G = G_;
  static constexpr int kStep = 1;
  static constexpr int kValues = 4;
  static constexpr int kHeadBytes = kTileBytes;
  static constexpr int kSliceWaves = 4;      // slices of a workgroup (one per compute unit)
  // s_waitcnt vmcnt(16): all but the loads of a step (12) and of query rows (4).
  static constexpr int kWaitOneStep = 0x4F70;
  struct Tile {
    bf16x8_t k[4];
    s16x4_t v[8];
  };
  struct Q {
    bf16x8_t f[4];
  };
  __device__ static int head(int lane) { return lane & 15; }
  __device__ static void load_q(Q& q, const uint16_t* __restrict__ rows, int lane) {
    const int h = head(lane), rq = lane >> 4;
    const uint16_t* row = rows + (h < G ? h : 0) * kHeadDim;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
      q.f[kb] = *reinterpret_cast<const bf16x8_t*>(row + kPiece * (4 * kb + rq));
  }
  template <bool kK, bool kV>
  __device__ static void load(Tile& x, int, const ShapedParams& p, size_t off, int lane) {
    if constexpr (kK) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
        x.k[kb] = stream_load<bf16x8_t>(p.k + off + 2 * kPiece * kWave * kb, 2 * kPiece * lane);
    }
    if constexpr (kV) {
      const int col = lane & 15, rq = lane >> 4;
#pragma unroll
      for (int mb = 0; mb < 8; ++mb)
        x.v[mb] = stream_load<s16x4_t>(p.v + off + 2 * 16 * kBlock * mb,
                                       2 * (col * kBlock + 4 * rq));
    }
  }
  __device__ static void scores(const Tile& x, const Q& q, float (&s)[kValues], int) {
    f32x4_t a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
      a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.k[kb], q.f[kb], a, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = a[i];
  }
  // First token of the four in s[4v .. 4v + 3].
  __device__ static int32_t position(int, const int32_t (&first)[kStep], int lane) {
    return first[0] + 4 * (lane >> 4);
  }
  __device__ static void hide_value(Tile& x, int, int i) {
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) x.v[mb][i] = 0;
  }
  __device__ static float head_max(float v) { return max_over_rows(v); }
  __device__ static float head_sum(float v) { return sum_over_rows(v); }
  __device__ static void add_values(f32x4_t (&acc)[8], const Tile& x, const float (&w)[kValues],
                                    int) {
    uint32_t q[3][2];
    split_weights(w, q);
    s16x4_t part[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const uint64_t two = (uint64_t)q[k][1] << 32 | q[k][0];
      part[k] = __builtin_bit_cast(s16x4_t, two);
    }
#pragma unroll
    for (int mb = 0; mb < 8; ++mb)
#pragma unroll
      for (int k = 0; k < 3; ++k)
        acc[mb] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(x.v[mb], part[k], acc[mb], 0, 0, 0);
  }
  __device__ static void fold(f32x4_t (&)[8]) {}
  // Word c (dims 4c .. 4c + 3) of this lane's head, for its eight words.
  template <class Fn>
  __device__ static void each_word(const f32x4_t (&acc)[8], int lane, Fn fn) {
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) fn(4 * mb + (lane >> 4), acc[mb]);
  }
};

// Packed: four blocks a step (64 tokens, 8.5 KiB, as much as a bf16 block), so
// that the running maximum, the rescaling and the addresses are paid once for 64
// tokens. Records become bf16 in registers, a pair of values an instruction.
//
// With up to eight heads a matrix product's 16 columns hold them twice. Of the scores
// of two blocks, lanes of columns 0-7 keep the first block's and those of columns 8-15
// the second's, so that half as many are left to each lane. The weights are sums of three
// bf16 numbers, as over bf16 caches: in one product columns 0-7 carry the first ones and
// 8-15 the second ones of both blocks (the lanes exchange what the other needs with a
// rotation by eight), in another the third ones, of the first block in columns 0-7 and of
// the second in 8-15, zeros beside them; the two halves of the sums are added in the end.
template <int G_>
struct PackedCache {
  static constexpr int G = G_;
  static constexpr int kStep = 4;
  static constexpr bool kTwice = G <= 8;
  static constexpr int kValues = kTwice ? 8 : 16;
  static constexpr int kHeadBytes = kPackedRecord;
  static constexpr int kSliceWaves = 8;
  static constexpr int kWaitOneStep = 0x4F74;  // vmcnt(20): 16 and 4
  struct Tile {
    u32x4_t k[kStep], v[kStep];
    uint32_t ke[kStep], ve[kStep];  // exponent bytes: of the K run, of four V tokens
  };
  struct Q {
    bf16x8_t f[4];
  };
  __device__ static int head(int lane) { return lane & (kTwice ? 7 : 15); }
  __device__ static void load_q(Q& q, const uint16_t* __restrict__ rows, int lane) {
    const int h = head(lane), rq = lane >> 4;
    const uint16_t* row = rows + (h < G ? h : 0) * kHeadDim;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
      q.f[kb] = *reinterpret_cast<const bf16x8_t*>(row + kScaleGroup * rq + 8 * kb);
  }
  template <bool kK, bool kV>
  __device__ static void load(Tile& x, int u, const ShapedParams& p, size_t off, int lane) {
    const uint8_t* rec = p.k + off;
    if constexpr (kK) {
      x.k[u] = stream_load<u32x4_t>(rec, 16 * lane);
      x.ke[u] = stream_load<uint8_t>(rec + kPackedKExp, lane);
    }
    if constexpr (kV) {
      x.v[u] = stream_load<u32x4_t>(rec + kPackedV, 16 * lane);
      x.ve[u] =
          stream_load<uint32_t>(rec + kPackedVExp, 16 * (lane >> 4) + 4 * ((lane & 15) >> 2));
    }
  }
  __device__ static float scale_of(uint32_t exponent) {
    return __builtin_bit_cast(float, exponent << 23);
  }
  // Of byte i of four. The conversions read a scale's exponent alone, so what the other
  // bytes leave in its sign and mantissa does not matter.
  __device__ static float scale_of_byte(uint32_t exponents, int i) {
    return __builtin_bit_cast(float, i < 3 ? exponents << (23 - 8 * i) : exponents >> 1);
  }
  // Eight 4-bit numbers times their scale.
  __device__ static bf16x8_t eight(uint32_t word, float scale) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0);
    const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2);
    const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3);
    const u32x4_t r = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                       __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
    return __builtin_bit_cast(bf16x8_t, r);
  }
  __device__ static void scores(const Tile& x, const Q& q, float (&s)[kValues], int lane) {
    f32x4_t a[kStep];
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      a[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const float scale = scale_of(x.ke[u]);
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
        a[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight(x.k[u][kb], scale), q.f[kb], a[u], 0,
                                                       0, 0);
    }
    const bool second = lane & 8;
#pragma unroll
    for (int v = 0; v < kValues; ++v) {
      if constexpr (kTwice)
        s[v] = second ? a[2 * (v / 4) + 1][v % 4] : a[2 * (v / 4)][v % 4];
      else
        s[v] = a[v / 4][v % 4];
    }
  }
  __device__ static int32_t position(int v, const int32_t (&first)[kStep], int lane) {
    if constexpr (kTwice) {
      const int32_t a = first[2 * v], b = first[2 * v + 1];
      return (lane & 8 ? b : a) + 4 * (lane >> 4);
    } else {
      return first[v] + 4 * (lane >> 4);
    }
  }
  // A record may hold anything where no token was written, NaN among it: its
  // numbers and their exponent are both replaced.
  __device__ static void hide_value(Tile& x, int u, int i) {
    x.v[u][i] = 0;
    x.ve[u] = (x.ve[u] & ~(0xFFu << (8 * i))) | (127u << (8 * i));
  }
  __device__ static float head_max(float v) {
    v = max_over_rows(v);
    return kTwice ? fmaxf(v, from_xor8(v)) : v;
  }
  __device__ static float head_sum(float v) {
    v = sum_over_rows(v);
    return kTwice ? v + from_xor8(v) : v;
  }
  __device__ static void add_values(f32x4_t (&acc)[8], const Tile& x, const float (&w)[kValues],
                                    int lane) {
    const bool second = lane & 8;
#pragma unroll
    for (int pair = 0; pair < kStep / 2; ++pair) {
      // Weights of the two blocks: four tokens of each, two to a register, in three parts.
      u32x4_t part[3];
      if constexpr (kTwice) {
        uint32_t q[3][2];
        split_weights(w + 4 * pair, q);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          part[0][i] = upper_from_xor8(q[0][i], q[1][i]);
          part[0][2 + i] = lower_from_xor8(q[1][i], q[0][i]);
          part[1][i] = second ? 0 : q[2][i];
          part[1][2 + i] = second ? q[2][i] : 0;
        }
      } else {
        uint32_t q[3][2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          split_weights(w + 8 * pair + 4 * b, q);
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            part[k][2 * b] = q[k][0];
            part[k][2 * b + 1] = q[k][1];
          }
        }
      }
      float scale[2][4];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          scale[b][i] = scale_of_byte(x.ve[2 * pair + b], i);
      auto product = [&](int m, const u32x4_t& a) {
#pragma unroll
        for (int k = 0; k < (kTwice ? 2 : 3); ++k)
          acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                           __builtin_bit_cast(bf16x8_t, part[k]),
                                                           acc[m], 0, 0, 0);
      };
      // Dims 2j and 2j + 1 of the lane's octet: a pair of dims of each token
      // becomes a pair of tokens of each dim.
      auto dims = [&](int m, auto conv) {
        u32x4_t even, odd;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t t0 = conv(x.v[2 * pair + b][2 * i], scale[b][2 * i]);
            const uint32_t t1 = conv(x.v[2 * pair + b][2 * i + 1], scale[b][2 * i + 1]);
            even[2 * b + i] = __builtin_amdgcn_perm(t1, t0, 0x05040100);
            odd[2 * b + i] = __builtin_amdgcn_perm(t1, t0, 0x07060302);
          }
        product(m, even);
        product(m + 1, odd);
      };
      dims(0, [](uint32_t a, float f) { return pair_of<0>(a, f); });
      dims(2, [](uint32_t a, float f) { return pair_of<1>(a, f); });
      dims(4, [](uint32_t a, float f) { return pair_of<2>(a, f); });
      dims(6, [](uint32_t a, float f) { return pair_of<3>(a, f); });
    }
  }
  template <int kByte>
  __device__ static uint32_t pair_of(uint32_t word, float scale) {
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, kByte));
  }
  __device__ static void fold(f32x4_t (&acc)[8]) {
    if constexpr (kTwice) {
#pragma unroll
      for (int m = 0; m < 8; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][i] += from_xor8(acc[m][i]);
    }
  }
  // acc[m][i] is dim 8 (4 rq + i) + m.
  template <class Fn>
  __device__ static void each_word(const f32x4_t (&acc)[8], int lane, Fn fn) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int half = 0; half < 2; ++half)
        fn(2 * (4 * (lane >> 4) + i) + half,
           f32x4_t{acc[4 * half][i], acc[4 * half + 1][i], acc[4 * half + 2][i],
                   acc[4 * half + 3][i]});
  }
};

// ------------------------------------------------------------------ a step

// A request and kv head with what the request sees; the same in all lanes.
struct Place {
  int32_t b, g;
  Seen seen;
};
// The pair's query rows and biases, as a lane holds them.
template <class C>
struct Pair {
  typename C::Q q;
  // Distances are counted from the token of this head's largest bias, so that
  // the biases that matter are small numbers.
  float slope_log2;
  int32_t origin;
};

template <class C>
__device__ inline void set_bias(const ShapedParams& p, const Place& at, Pair<C>& pr, int lane) {
  const int h = C::head(lane);
  const float slope = p.slopes && h < C::G ? p.slopes[at.g * C::G + h] : 0.f;
  pr.slope_log2 = slope * 1.4426950408889634f;
  pr.origin = slope >= 0.f ? at.seen.L - 1 : at.seen.first();
}
template <class C>
__device__ inline Pair<C> make_pair(const ShapedParams& p, const Place& at, int lane) {
  Pair<C> pr;
  set_bias<C>(p, at, pr, lane);
  C::load_q(pr.q, p.q + ((size_t)at.b * p.hq + at.g * C::G) * kHeadDim, lane);
  return pr;
}
// The bias of token `origin`, which the scores leave out (natural units): its
// slope times a distance.
template <class C>
__device__ inline float left_out(const ShapedParams& p, int32_t g, int h, const Seen& seen) {
  if (!p.slopes) return 0.f;
  const float slope = p.slopes[g * C::G + h];
  return slope >= 0.f ? 0.f : slope * (float)(seen.first() - (seen.L - 1));
}

// The physical blocks of step j: of virtual blocks kStep j .., and the last one again
// where there are no more (its tokens count for nothing there).
template <class C>
struct Blocks {
  int32_t id[C::kStep];
};
template <class C>
__device__ inline Blocks<C> find_blocks(const ShapedParams& p, const Place& at, int32_t j) {
  Blocks<C> r;
  const ScalarInts row = scalar_ints(p.table) + (size_t)at.b * p.mbps;
  const Seen& seen = at.seen;
  const int32_t v0 = j * C::kStep;
  if (v0 + C::kStep <= seen.n && (v0 >= seen.pb || v0 + C::kStep <= seen.pb)) {
    const ScalarInts ids = row + seen.block_of(v0);  // a run of the table
#pragma unroll
    for (int u = 0; u < C::kStep; ++u) r.id[u] = ids[u];
  } else {
#pragma unroll
    for (int u = 0; u < C::kStep; ++u) r.id[u] = row[seen.block_of(min(v0 + u, seen.n - 1))];
  }
  return r;
}
// First tokens of the step's blocks; where there is no block, a token that nobody sees.
constexpr int32_t kNoToken = 0x7FFFFF00;
template <class C>
__device__ inline void first_tokens(const Seen& seen, int32_t j, int32_t (&first)[C::kStep]) {
#pragma unroll
  for (int u = 0; u < C::kStep; ++u) {
    const int32_t v = j * C::kStep + u;
    first[u] = v < seen.n ? seen.block_of(v) * kBlock : kNoToken;
  }
}

template <class C, bool kK, bool kV>
__device__ inline void load_step(const ShapedParams& p, const Place& at, const Blocks<C>& blocks,
                                 typename C::Tile& t, int lane) {
  // (Keeps the lanes' offsets from being widened to 64 bits ahead of a loop, which costs an
  // addition a load in it: a load adds 32 bits to a uniform base itself.)
  asm volatile("" : "+v"(lane));
#pragma unroll
  for (int u = 0; u < C::kStep; ++u) {
    const uint32_t id = min((uint32_t)blocks.id[u], (uint32_t)(p.num_blocks - 1));
    C::template load<kK, kV>(t, u, p,
                             (size_t)id * (size_t)p.blk_bytes + (size_t)(at.g * C::kHeadBytes),
                             lane);
  }
}

// A step's products q.k become its scores, in base 2 and without the bias of the pair's
// origin: x times the factor returned (that of plain scores is left to be multiplied
// where the maximum is subtracted).
template <class C>
__device__ inline float shape_scores(const ShapedParams& p, const Seen& seen, const Pair<C>& pr,
                                    const int32_t (&first)[C::kStep], bool all,
                                    float (&x)[C::kValues], int lane) {
  float factor = 1.f;
  if (p.cap_log2 != 0.f) {
    // Caps are mostly far above the scores: where all of a wavefront's are small the
    // exponentials are passed over (a window of 1500 tokens, capped at 50: 212 -> 208 us; packed
    // weight sums 69.5 -> 67.8). A NaN is neither, and stays one.
    float largest = 0.f;
#pragma unroll
    for (int v = 0; v < C::kValues; ++v) {
      x[v] *= p.cap_in;
      largest = fmaxf(largest, fabsf(x[v]));
    }
    if (__any(largest >= kSmallTanh)) {
#pragma unroll
      for (int v = 0; v < C::kValues; ++v) x[v] = p.cap_log2 * any_tanh(x[v]);
    } else {
#pragma unroll
      for (int v = 0; v < C::kValues; ++v) x[v] = p.cap_log2 * small_tanh(x[v]);
    }
  } else if (!p.slopes && p.scale_log2 > 0.f) {
    factor = p.scale_log2;
  } else {
#pragma unroll
    for (int v = 0; v < C::kValues; ++v) x[v] *= p.scale_log2;
  }
  if (p.slopes) {
#pragma unroll
    for (int v = 0; v < C::kValues; v += 4) {
      const int32_t d = C::position(v / 4, first, lane) - pr.origin;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[v + i] = fmaf(pr.slope_log2, (float)(d + i), x[v + i]);
    }
  }
  if (!all) {
#pragma unroll
    for (int v = 0; v < C::kValues; v += 4) {
      const int32_t t0 = C::position(v / 4, first, lane);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!seen.sees(t0 + i)) x[v + i] = -INFINITY;
    }
  }
  return factor;
}

// The running softmax of one head (and the sums of its lanes).
struct Softmax {
  f32x4_t acc[8];
  float m;  // maximum so far, the same in all lanes of a head
  float l;  // this lane's share of the denominator
  __device__ void init() {
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) acc[mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m = kLowest;
    l = 0.f;
  }
};

// A step's products x into the running softmax, with its values.
template <class C>
__device__ inline void attend_scores(const ShapedParams& p, const Seen& seen, const Pair<C>& pr,
                                     typename C::Tile& t, int32_t j, float (&x)[C::kValues],
                                     Softmax& st, int lane) {
  const bool all = seen.sees_all(j * C::kStep, C::kStep);
  int32_t first[C::kStep];
  first_tokens<C>(seen, j, first);
  const float factor = shape_scores<C>(p, seen, pr, first, all, x, lane);
  if (!all) {
#pragma unroll
    for (int u = 0; u < C::kStep; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!seen.sees(first[u] + 4 * (lane >> 4) + i)) C::hide_value(t, u, i);
  }
  float mt = x[0];
#pragma unroll
  for (int v = 1; v < C::kValues; ++v) mt = fmaxf(mt, x[v]);
  const float mn = fmaxf(st.m, C::head_max(mt) * factor);
  const float alpha = __builtin_amdgcn_exp2f(st.m - mn);
  float sum = 0.f;
#pragma unroll
  for (int v = 0; v < C::kValues; ++v) {
    x[v] = __builtin_amdgcn_exp2f(fmaf(x[v], factor, -mn));
    sum += x[v];
  }
  st.l = fmaf(st.l, alpha, sum);
  st.m = mn;
  // Maxima stop growing after a few steps.
  if (__any(alpha != 1.f)) {
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) st.acc[mb] *= alpha;
  }
  C::add_values(st.acc, t, x, lane);
}
template <class C>
__device__ inline void attend_step(const ShapedParams& p, const Seen& seen, const Pair<C>& pr,
                                   typename C::Tile& t, int32_t j, Softmax& st, int lane) {
  float x[C::kValues];
  // Ahead of the other wavefronts of a SIMD, which so come to stand at other places of
  // their steps (packed, 512 x U[256, 4096]: 227 -> 223 us; a window of 1500: 212 -> 210).
  __builtin_amdgcn_s_setprio(1);
  C::scores(t, pr.q, x, lane);
  __builtin_amdgcn_s_setprio(0);
  attend_scores<C>(p, seen, pr, t, j, x, st, lane);
}

// Steps j0, j0 + stride, ... below j1 of a pair: `load` requests a step's tile and `body`
// uses it, one step in flight ahead of the one computed and block ids another ahead.
template <class C, class Tile, class Load, class Body>
__device__ inline void each_step(const ShapedParams& p, const Place& pl, int32_t j0, int32_t j1,
                                 int32_t stride, Load load, Body body) {
  if (j0 >= j1) return;
  Tile t0, t1;
  load(t0, find_blocks<C>(p, pl, j0), j0);
  if (j0 + stride >= j1) return body(t0, j0);
  // (The last step stands outside of the loop, so that every step in it requests as much.)
  const int32_t last = j1 - 1;
  Blocks<C> ids = find_blocks<C>(p, pl, j0 + stride);
  for (int32_t j = j0;;) {
    load(t1, ids, j + stride);
    ids = find_blocks<C>(p, pl, min(j + 2 * stride, last));
    body(t0, j);
    j += stride;
    if (j + stride >= j1) return body(t1, j);
    load(t0, ids, j + stride);
    ids = find_blocks<C>(p, pl, min(j + 2 * stride, last));
    body(t1, j);
    j += stride;
    if (j + stride >= j1) return body(t0, j);
  }
}

}  // namespace neo
