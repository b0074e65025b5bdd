// Matrix products, operands in 8 bits.
#include <type_traits>

#include "matmul_impl.inc"

namespace dwm {
dwm_status_t launch_matmul_packed(const MatmulArgs& a, int flags, int kernel, void* stream) { return run_kernel<uint8_t>(a, flags, kernel, stream); }
}  // namespace dwm
