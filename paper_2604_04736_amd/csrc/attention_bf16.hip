// libhot: the kernels of attention.h for bfloat16.
#include "attention.h"

HOT_ATTENTION_OF(__bf16);
