#define ICONV_MAT_T __half
#define ICONV_MAT_ID 1
#include "mat_inst.cuh"
