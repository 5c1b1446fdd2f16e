// Products of E4M3 and E4M3 factors.
#define MAT_FA 0
#define MAT_FB 0
#include "vec_matmul_launch.h"
