// The attention kernels for f32 queries.
#include "attn8_kernel.h"

template ds::AttnKernel ds::attn8_kernel<float>(int form, int fmt, int stype, int dim, bool exact);
