// Attention with shaped scores over bf16 caches.
#include "shaped_kernels.h"
#include "shaped_ops.h"

namespace neo {

hipError_t launch_shaped_bf16(const ShapedParams& p, int32_t group, bool weights,
                              hipStream_t stream) {
  return launch_shaped<Bf16Cache>(p, group, weights, stream);
}

}  // namespace neo
