// Launch and opt-in functions of the product kernels' instances, one translation unit per output type (mat_inst0.cu float, 1 half, 2 bfloat16).
#pragma once

#include "mat_device.cuh"
#include "mat_stream.cuh"

namespace iconv {

struct MatLaunch {
    unsigned grid, threads;
    size_t smem;
    cudaStream_t stream;
    bool bulk, streams;             // the bulk kernel, the streaming kernel, else the few-tile kernel
    const CUtensorMap *tmap_w, *tmap_x;
    const MatArgs *a;
    const MatStreamArgs *s;
};

#define ICONV_DECLARE_MAT(E) cudaError_t mat_launch_##E(bool gated, const MatLaunch &l); cudaError_t mat_opt_in_##E();
ICONV_DECLARE_MAT(0) ICONV_DECLARE_MAT(1) ICONV_DECLARE_MAT(2)
#undef ICONV_DECLARE_MAT

}  // namespace iconv
