// The element type that a file of the gated delta rule is compiled for: bfloat16, or what it is included with.
#ifdef COTTN_DELTA_F16
#define DELTA_T _Float16
#define DELTA_SYM(name) name##_f16
#elif defined(COTTN_DELTA_F32)
#define DELTA_T float
#define DELTA_SYM(name) name##_f32
#else
#define DELTA_T __bf16
#define DELTA_SYM(name) name##_bf16
#endif
