// The norm kernels for binary16 tensors (norm_impl.inc).
#define NORM_T _Float16
#define NORM_LAUNCH launch_norm_f16
#include "norm_impl.inc"
