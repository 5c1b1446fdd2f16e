// Products of E4M3 and E5M2 factors.
#define MAT_FA 0
#define MAT_FB 1
#include "vec_matmul_launch.h"
