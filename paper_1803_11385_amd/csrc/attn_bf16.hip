// Attention kernels for bf16 operands.
#define HCH_ATTN_TYPE __bf16
#include "attn_launch.hpp"
