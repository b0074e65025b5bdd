// Matrix products, operands in bfloat16.
#include <type_traits>

#include "matmul_impl.inc"

namespace dwm {
dwm_status_t launch_matmul_bf16(const MatmulArgs& a, int flags, int kernel, void* stream) { return run_kernel<__bf16>(a, flags, kernel, stream); }
}  // namespace dwm
