#define CHOCO_LINEAR_TYPE bf16_t
#include "choco_linear_chunks.h"
