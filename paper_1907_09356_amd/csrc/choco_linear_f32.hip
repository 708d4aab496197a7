#define CHOCO_LINEAR_TYPE float
#include "choco_linear_chunks.h"
