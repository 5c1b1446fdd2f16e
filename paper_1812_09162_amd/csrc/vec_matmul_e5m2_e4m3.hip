// Products of E5M2 and E4M3 factors.
#define MAT_FA 1
#define MAT_FB 0
#include "vec_matmul_launch.h"
