#define CHOCO_LINEAR_TYPE f16_t
#include "choco_linear_chunks.h"
