// Launch and opt-in functions of the product kernels' instances, one translation unit per output type (mat_inst0.cu float, 1 half, 2 bfloat16).
#pragma once

#include "mat_device.cuh"

namespace iconv {

struct MatLaunch {
    unsigned grid;
    size_t smem;
    cudaStream_t stream;
    int split;                      // 0: the bulk kernel; else the few-token kernel's CTAs per tile (1, 2, 4 or 8)
    const CUtensorMap *tmap_w, *tmap_x;
    const MatArgs *a;
};

#define ICONV_DECLARE_MAT(E) cudaError_t mat_launch_##E(bool gated, const MatLaunch &l); cudaError_t mat_opt_in_##E();
ICONV_DECLARE_MAT(0) ICONV_DECLARE_MAT(1) ICONV_DECLARE_MAT(2)
#undef ICONV_DECLARE_MAT

}  // namespace iconv
