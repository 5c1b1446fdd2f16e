// Products of E5M2 and E5M2 factors.
#define MAT_FA 1
#define MAT_FB 1
#include "vec_matmul_launch.h"
