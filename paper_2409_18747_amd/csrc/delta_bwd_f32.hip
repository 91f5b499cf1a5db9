// The kernels of delta_bwd_bf16.hip for rows in fp32.
#define COTTN_DELTA_F32
#include "delta_bwd_bf16.hip"
