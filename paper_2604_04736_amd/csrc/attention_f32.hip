// libhot: the kernels of attention.h for float32.
#include "attention.h"

HOT_ATTENTION_OF(float);
