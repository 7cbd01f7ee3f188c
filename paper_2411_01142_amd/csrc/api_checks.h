// Argument checks and device facts shared by the C ABI's translation units. All
// checks run on the host before any HIP call.
#pragma once

#include <math.h>
#include <stdint.h>

#include <atomic>

#include "neo_error.h"
#include "neo_internal.h"

namespace neo {

inline neo_status ok() { return neo::clear_error(); }

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

inline bool supported_group(int32_t g) { return g == 1 || g == 2 || g == 4 || g == 8 || g == 16; }

// Compute units of the current device, cached per device ordinal. The default
// plan uses at most CUs x wavefronts per workgroup slices (one workgroup per
// CU).
constexpr int kMaxDevices = 64;
// Per device ordinal: compute units in the low 16 bits, XCDs above (0: not
// read yet).
inline std::atomic<int32_t> g_device_shape[kMaxDevices];

// Compute units and XCDs of the current device.
inline neo_status device_shape(int32_t* cus, int32_t* xcds) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return set_error(NEO_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
  if (dev >= 0 && dev < kMaxDevices) {
    const int32_t cached = g_device_shape[dev].load(std::memory_order_relaxed);
    if (cached > 0) {
      *cus = cached & 0xFFFF;
      *xcds = cached >> 16;
      return NEO_OK;
    }
  }
  int v = 0, x = 0;
  e = hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess || v <= 0 || v > 0xFFFF)
    return set_error(NEO_ERR_HIP, "hipDeviceGetAttribute(cu count): %s", hipGetErrorString(e));
  // An XCD count the runtime cannot give only turns the slice weights off.
  if (hipDeviceGetAttribute(&x, hipDeviceAttributeNumberOfXccs, dev) != hipSuccess || x < 1 ||
      x > 0x7FFF) {
    (void)hipGetLastError();
    x = 1;
  }
  if (dev >= 0 && dev < kMaxDevices)
    g_device_shape[dev].store(v | (x << 16), std::memory_order_relaxed);
  *cus = v;
  *xcds = x;
  return NEO_OK;
}

inline neo_status check_heads(int32_t hq, int32_t hkv, int32_t head_dim) {
  if (hq <= 0 || hkv <= 0)
    return set_error(NEO_ERR_INVALID_ARG, "num_q_heads (%d) and num_kv_heads (%d) must be positive",
                     hq, hkv);
  if (hq % hkv != 0)
    return set_error(NEO_ERR_INVALID_ARG, "num_q_heads (%d) is not a multiple of num_kv_heads (%d)",
                     hq, hkv);
  if (head_dim != neo::kHeadDim)
    return set_error(NEO_ERR_UNSUPPORTED, "head_dim %d unsupported (only %d)", head_dim,
                     neo::kHeadDim);
  if (!supported_group(hq / hkv))
    return set_error(NEO_ERR_UNSUPPORTED, "query group %d unsupported (1, 2, 4, 8 or 16)",
                     hq / hkv);
  return NEO_OK;
}

// A cache's block stride in elements: 0 stands for `dense` (num_kv_heads tiles,
// blocks back to back); otherwise a multiple of 8 (whole 16-byte words) of at
// least `dense` -- the stride may leave room after a block (the other cache's
// block, padding) but not less -- and at most 2^40, so that block id * stride
// stays far inside 64 bits. *resolved gets the stride to use.
inline neo_status check_block_stride(int64_t stride, int64_t dense, const char* name,
                              int64_t* resolved) {
  if (stride != 0 &&
      (stride < dense || stride % neo::kPiece != 0 || stride > ((int64_t)1 << 40)))
    return set_error(NEO_ERR_INVALID_ARG,
                     "%s %lld must be 0 or a multiple of %d of at least %lld elements "
                     "(and at most 2^40)",
                     name, (long long)stride, neo::kPiece, (long long)dense);
  *resolved = stride != 0 ? stride : dense;
  return NEO_OK;
}

// The caches' byte span (num_blocks blocks at `stride` elements) must stay far
// inside 64 bits, so that no block offset the kernels form can wrap.
inline neo_status check_span(int64_t stride, int32_t num_blocks, const char* name) {
  if (num_blocks > 0 && stride > (((int64_t)1 << 61) / num_blocks))
    return set_error(NEO_ERR_INVALID_ARG,
                     "%s: %d blocks at a stride of %lld elements span 2^62 bytes or more",
                     name, num_blocks, (long long)stride);
  return NEO_OK;
}

}  // namespace neo
