// The attention kernels for f32 queries.
#include "attn8_kernel.h"

template const void *ds::attn8_kernel<float>(int fmt, int dim, bool few);
