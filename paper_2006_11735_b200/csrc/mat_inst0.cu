#define ICONV_MAT_T float
#define ICONV_MAT_ID 0
#include "mat_inst.cuh"
