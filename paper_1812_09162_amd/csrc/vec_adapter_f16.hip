// vec_adapter and vec_adapter_grad: the kernels for this type of matrices.
#define VEC_ADAPTER_SOURCE _Float16
#include "vec_adapter_launch.h"
