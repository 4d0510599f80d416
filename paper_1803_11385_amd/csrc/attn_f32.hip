// Attention kernels for fp32 operands.
#define HCH_ATTN_TYPE float
#include "attn_launch.hpp"
