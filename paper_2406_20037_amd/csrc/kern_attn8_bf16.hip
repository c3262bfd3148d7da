// The attention kernels for bf16 queries.
#include "attn8_kernel.h"

template ds::AttnKernel ds::attn8_kernel<__bf16>(int form, int fmt, int stype, int dim, bool exact);
