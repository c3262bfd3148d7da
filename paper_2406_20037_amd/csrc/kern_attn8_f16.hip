// The attention kernels for f16 queries.
#include "attn8_kernel.h"

template const void *ds::attn8_kernel<_Float16>(int fmt, int dim, bool few);
