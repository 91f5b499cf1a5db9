// The bwd decay kernels for fp32 elements, on the fp32 matrix instruction (see device_common.h).
#define COTTN_ELEM_F32
#define COTTN_F32_WHOLE
#include "bwd_decay_bf16.hip"
