// dsvt_set_mha on bf16 rows (see mha_forward.h).
#include "mha_forward.h"

int mha_forward_bf16(const MhaArgs& a, TableForm form, size_t lds, hipStream_t st) { return launch<bf16_t>(a, form, lds, st); }
