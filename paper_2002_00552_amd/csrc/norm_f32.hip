// The norm kernels for binary32 tensors (norm_impl.inc).
#define NORM_T float
#define NORM_LAUNCH launch_norm_f32
#include "norm_impl.inc"
