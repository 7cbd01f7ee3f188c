// Writing new tokens into a packed cache, and reading tokens back as bf16.
#include "decode_common.h"
#include "packed.h"
#include "shaped_ops.h"

namespace neo {
namespace {

// A workgroup takes 16 rows of one kv head, which in a prompt are a block or parts
// of two, so that the bytes of a record's lines meet in one L2; 16 threads a row,
// 8 dims each. Prompts are bound by HBM (five of 1000 to 6000 tokens, 8 kv heads: written
// 18.6 us, read back 15.5, 4.3 and 5.2 TB/s); a token for each of 256 requests by latency
// (3.2 and 2.8 us).
constexpr int kRowsPerGroup = 16;
constexpr int kRowThreads = kHeadDim / 8;

struct RowPlace {
  int64_t at;  // record's byte offset, or -1: no such token
  int slot;
};

// Where row r belongs. Every lane of the wavefront takes part; rows of a wavefront
// may differ. The request is the number of row_starts[1 ..] at or below r.
__device__ inline RowPlace find_row(const PackedRows& p, int32_t r, int32_t g, bool clamp_id) {
  const int lane = threadIdx.x & (kWave - 1);
  int32_t b = r, back = 1;  // rows from r to the end of its request
  bool found = r < p.rows;
  if (p.row_starts) {
    b = 0;
    for (int32_t base = 0; base < p.batch; base += kWave) {
      const int32_t e = base + lane < p.batch ? p.row_starts[base + lane + 1] : 0x7FFFFFFF;
#pragma unroll
      for (int k = 0; k < kWave / kRowThreads; ++k) {
        const int32_t rk = __builtin_amdgcn_readlane(r, k * kRowThreads);
        const int c = __popcll(__ballot(e <= rk));
        if (lane / kRowThreads == k) b += c;
      }
    }
    found = found && b < p.batch;
    if (found) {
      back = p.row_starts[b + 1] - r;
      found = r >= p.row_starts[b] && back > 0;
    }
  }
  RowPlace w{-1, 0};
  if (!found || b >= p.batch) return w;
  const int32_t t = clamp_len(p.lens[b], p.mbps) - back;
  if (t < 0) return w;
  int32_t blk = p.table[(size_t)b * p.mbps + t / kBlock];
  if (clamp_id) blk = (int32_t)min((uint32_t)blk, (uint32_t)(p.num_blocks - 1));
  if (blk < 0 || blk >= p.num_blocks) return w;
  w.at = (int64_t)blk * p.blk_bytes + (int64_t)g * kPackedRecord;
  w.slot = t % kBlock;
  return w;
}

// Maximum over each four neighbouring lanes, the 32 dims that share an exponent.
__device__ inline uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
}

struct PackedEight {
  uint32_t word, exponent;
};
// Eight bf16 values of a lane as 4-bit numbers, and the exponent byte of its group:
// from the largest magnitude's bits, its exponent less two, or less one from 1.75
// times a power of two on.
__device__ inline PackedEight pack_eight(const u32x4_t& x) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7FFFu, (x[i] >> 16) & 0x7FFFu));
  top = quad_max(top);
  const int32_t e = (int32_t)(top >> 7);
  int32_t byte = min(max(e - 2 + ((top & 0x7F) >= 0x60 ? 1 : 0), 2), 252);
  if (top == 0) byte = 0;
  if (e == 255) byte = 255;
  const float scale = __builtin_bit_cast(float, (uint32_t)byte << 23);
  // (Words are copied to scalars before the bit casts: a cast applied to a
  // vector-element subscript directly has been lowered as a read of element 0.)
  const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x0), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x1), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x2), scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x3), scale, 3);
  return {w, (uint32_t)byte};
}

__global__ __launch_bounds__(kRowsPerGroup* kRowThreads) void packed_append_kernel(
    PackedRows p, const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
    RowStrides s) {
  const int32_t g = blockIdx.x % p.hkv;
  const int32_t r = (int32_t)(blockIdx.x / p.hkv) * kRowsPerGroup + (int32_t)threadIdx.x / kRowThreads;
  const int octet = threadIdx.x % kRowThreads;
  // The values do not wait for the place.
  u32x4_t k = {0u, 0u, 0u, 0u}, v = k;
  if (r < p.rows) {
    k = *reinterpret_cast<const u32x4_t*>(k_new + r * s.k_row + g * s.k_head + 8 * octet);
    v = *reinterpret_cast<const u32x4_t*>(v_new + r * s.v_row + g * s.v_head + 8 * octet);
  }
  const RowPlace w = find_row(p, r, g, false);
  const PackedEight pk = pack_eight(k), pv = pack_eight(v);
  if (w.at < 0) return;
  uint8_t* rec = p.cache + w.at;
  *reinterpret_cast<uint32_t*>(rec + packed_k_at(w.slot, octet)) = pk.word;
  *reinterpret_cast<uint32_t*>(rec + packed_v_at(w.slot, octet)) = pv.word;
  if (octet % 4 == 0) {
    rec[packed_k_exp_at(w.slot, octet / 4)] = (uint8_t)pk.exponent;
    rec[packed_v_exp_at(w.slot, octet / 4)] = (uint8_t)pv.exponent;
  }
}

__device__ inline u32x4_t unpack_eight(uint32_t word, uint32_t exponent) {
  const float scale = __builtin_bit_cast(float, exponent << 23);
  return u32x4_t{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3))};
}

__global__ __launch_bounds__(kRowsPerGroup* kRowThreads) void packed_gather_kernel(
    PackedRows p, uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out) {
  const int32_t g = blockIdx.x % p.hkv;
  const int32_t r = (int32_t)(blockIdx.x / p.hkv) * kRowsPerGroup + (int32_t)threadIdx.x / kRowThreads;
  const int octet = threadIdx.x % kRowThreads;
  const RowPlace w = find_row(p, r, g, true);
  if (w.at < 0) return;
  const uint8_t* rec = p.cache + w.at;
  const uint32_t k = *reinterpret_cast<const uint32_t*>(rec + packed_k_at(w.slot, octet));
  const uint32_t v = *reinterpret_cast<const uint32_t*>(rec + packed_v_at(w.slot, octet));
  const size_t dst = ((size_t)r * p.hkv + g) * kHeadDim + 8 * octet;
  *reinterpret_cast<u32x4_t*>(k_out + dst) =
      unpack_eight(k, rec[packed_k_exp_at(w.slot, octet / 4)]);
  *reinterpret_cast<u32x4_t*>(v_out + dst) =
      unpack_eight(v, rec[packed_v_exp_at(w.slot, octet / 4)]);
}

unsigned row_groups(const PackedRows& p) {
  return (unsigned)(((int64_t)p.rows + kRowsPerGroup - 1) / kRowsPerGroup * p.hkv);
}

}  // namespace

hipError_t launch_packed_append(const PackedRows& p, const uint16_t* k_new, const uint16_t* v_new,
                                const RowStrides& s, hipStream_t stream) {
  packed_append_kernel<<<row_groups(p), kRowsPerGroup * kRowThreads, 0, stream>>>(p, k_new, v_new,
                                                                                  s);
  return hipGetLastError();
}

hipError_t launch_packed_gather(const PackedRows& p, uint16_t* k_out, uint16_t* v_out,
                                hipStream_t stream) {
  packed_gather_kernel<<<row_groups(p), kRowsPerGroup * kRowThreads, 0, stream>>>(p, k_out, v_out);
  return hipGetLastError();
}

}  // namespace neo
