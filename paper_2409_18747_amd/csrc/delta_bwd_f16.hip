// The kernels of delta_bwd_bf16.hip for rows in IEEE half precision.
#define COTTN_DELTA_F16
#include "delta_bwd_bf16.hip"
