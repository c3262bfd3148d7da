// The attention kernels for bf16 queries.
#include "attn8_kernel.h"

template const void *ds::attn8_kernel<__bf16>(int fmt, int dim, bool few);
