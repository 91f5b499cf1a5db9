// The kernels of delta_fwd_bf16.hip for rows in IEEE half precision.
#define COTTN_DELTA_F16
#include "delta_fwd_bf16.hip"
