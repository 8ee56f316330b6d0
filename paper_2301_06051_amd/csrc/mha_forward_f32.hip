// dsvt_set_mha on fp32 rows (see mha_forward.h).
#include "mha_forward.h"

int mha_forward_f32(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st) { return launch<float>(a, form, lds, st); }
