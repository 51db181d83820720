// The experts' products on 4-bit codes.
#define QG_EXPERTS_KERNELS
#include "qg_experts_few.h"

void qg_few_launch_b4(const QgFewArgs &f, hipStream_t st) { few_launch<4>(f, st); }
