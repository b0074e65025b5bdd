// The norm kernels for bfloat16 tensors (norm_impl.inc).
#define NORM_T __bf16
#define NORM_LAUNCH launch_norm_bf16
#include "norm_impl.inc"
