#define ICONV_MAT_T __nv_bfloat16
#define ICONV_MAT_ID 2
#include "mat_inst.cuh"
