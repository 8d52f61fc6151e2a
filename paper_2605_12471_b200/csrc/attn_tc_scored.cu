// The tcgen05 attention kernels of scored steps (attn_tc.cu has the kernel, and the plain ones).
#define KVF_SCORED_KERNELS
#include "attn_tc.cu"
