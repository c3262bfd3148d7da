// The attention kernels for f16 queries.
#include "attn8_kernel.h"

template ds::AttnKernel ds::attn8_kernel<_Float16>(int form, int fmt, int stype, int dim, bool exact);
