// libhot: the kernels of attention.h for float16.
#include "attention.h"

HOT_ATTENTION_OF(_Float16);
