// The experts' products on 2-bit codes.
#include <atomic>

#define QG_EXPERTS_KERNELS
#include "qg_experts_few.h"
#include "qg_experts_many.h"

void qg_few_launch_b2(const QgFewArgs &f, const QgPrepareArgs &p, hipStream_t st) { few_launch<2>(f, p, st); }
int qg_many_launch_b2(const QgManyArgs &f, const QgPrepareArgs &p, hipStream_t st) { return many_launch<2>(f, p, st); }
