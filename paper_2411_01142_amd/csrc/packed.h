// The 4-bit ("packed") KV cache: layout of a record, the K and V of one block of
// 16 tokens and one kv head, and the rule by which values become 4-bit numbers.
//
// Values are e2m1 numbers (a sign; 0, 0.5, 1, 1.5, 2, 3, 4 or 6) times a power
// of two that 32 consecutive dims of a token share, the microscaling fp4 format,
// which gfx950 converts in hardware: both directions are one instruction for
// two values, and a number times its power of two is exact in bf16, so the
// matrix cores read exactly the values that the record stands for. 136 bytes for
// K and V of a token and kv head, 0.27 of bf16's 512.
//
// The exponent e of 32 values with largest magnitude a is the smallest with
// a < 7 * 2^e: a then rounds to at most 6 * 2^e, and the largest value is off by
// no more than half of the step there, like any other (with the exponent that
// brings a below 8 * 2^e, values between 7 and 8 are cut to 6; with 6 * 2^e, the
// others lose a bit for them more often). e is kept in [-125, 125], where every product is a
// normal finite bf16. The byte stored is e + 127; 0 for a group of zeros, 255
// (every value NaN) for a group that holds an infinity or a NaN.
//
// A record's 2176 bytes, every part in the order in which a wavefront's lanes
// load it (lane l: row l % 16, group l / 16):
//   K        [4 dim groups][16 tokens][16 bytes]          byte j: dims 2j, 2j + 1
//   V        [4 token groups][16 dim octets][4 tokens][4 bytes]         likewise
//   K exp.   [4 dim groups][16 tokens]
//   V exp.   [4 token groups][4 dim groups][4 tokens]
// A lane's 16 bytes of K are the 32 dims that share its exponent byte, one dword
// for each of the four matrix products of a block. Its 16 bytes of V are eight
// dims of four tokens. Every token has bytes of its own, so tokens are written
// without reading their neighbours.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace neo {

constexpr int kScaleGroup = 32;      // dims that share an exponent
constexpr int kPackedV = 1024;       // byte offsets in a record
constexpr int kPackedKExp = 2048;
constexpr int kPackedVExp = 2112;
constexpr int kPackedRecord = 2176;

// Byte of a token's K (V) that holds the 8 dims from 8 * octet on.
__host__ __device__ inline int packed_k_at(int slot, int octet) {
  return (octet / 4) * 256 + slot * 16 + (octet % 4) * 4;
}
__host__ __device__ inline int packed_v_at(int slot, int octet) {
  return kPackedV + (slot / 4) * 256 + octet * 16 + (slot % 4) * 4;
}
// Byte of its exponent for dims 32 * group .. + 31.
__host__ __device__ inline int packed_k_exp_at(int slot, int group) {
  return kPackedKExp + group * 16 + slot;
}
__host__ __device__ inline int packed_v_exp_at(int slot, int group) {
  return kPackedVExp + (slot / 4) * 16 + group * 4 + slot % 4;
}

}  // namespace neo
