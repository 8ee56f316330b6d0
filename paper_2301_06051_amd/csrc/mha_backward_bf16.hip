// dsvt_set_mha_backward on bf16 rows (see mha_backward.h).
#include "mha_backward.h"

int mha_backward_bf16(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st) { return launch<bf16_t>(a, form, lds, st); }
