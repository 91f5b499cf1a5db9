// The kernels of delta_fwd_bf16.hip for rows in fp32.
#define COTTN_DELTA_F32
#include "delta_fwd_bf16.hip"
