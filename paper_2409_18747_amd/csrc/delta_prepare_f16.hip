// The kernels of delta_prepare_bf16.hip for rows in IEEE half precision.
#define COTTN_DELTA_F16
#include "delta_prepare_bf16.hip"
