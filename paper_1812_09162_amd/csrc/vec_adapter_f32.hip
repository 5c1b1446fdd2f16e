// vec_adapter and vec_adapter_grad: the kernels for this type of matrices.
#define VEC_ADAPTER_SOURCE float
#include "vec_adapter_launch.h"
