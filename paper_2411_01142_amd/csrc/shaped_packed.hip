// Attention (with shaped scores) over packed caches.
#include "shaped_kernels.h"
#include "shaped_ops.h"

namespace neo {

hipError_t launch_shaped_packed(const ShapedParams& p, int32_t group, bool weights,
                                hipStream_t stream) {
  return launch_shaped<PackedCache>(p, group, weights, stream);
}

}  // namespace neo
