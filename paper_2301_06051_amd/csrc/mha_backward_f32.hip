// dsvt_set_mha_backward on fp32 rows (see mha_backward.h).
#include "mha_backward.h"

int mha_backward_f32(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st) { return launch<float>(a, form, lds, st); }
