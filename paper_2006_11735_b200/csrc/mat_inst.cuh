// Body of one translation unit of product kernels: define ICONV_MAT_T (output type) and ICONV_MAT_ID before including.
#include "mat_inst.h"

namespace iconv {

#define ICONV_CAT2(a, b) a##b
#define ICONV_CAT(a, b) ICONV_CAT2(a, b)

namespace {

using MatKernel = void (*)(CUtensorMap, CUtensorMap, MatArgs);

MatKernel instance(bool gated, bool bulk)
{
    if (bulk) return gated ? mat_bulk_kernel<ICONV_MAT_T, true> : mat_bulk_kernel<ICONV_MAT_T, false>;
    return gated ? mat_few_kernel<ICONV_MAT_T, true> : mat_few_kernel<ICONV_MAT_T, false>;
}

using MatStreamKernel = void (*)(MatStreamArgs, MatArgs);

MatStreamKernel stream_instance(bool gated, bool wide)
{
    if (wide) return gated ? mat_stream_kernel<ICONV_MAT_T, true, 2> : mat_stream_kernel<ICONV_MAT_T, false, 2>;
    return gated ? mat_stream_kernel<ICONV_MAT_T, true, 1> : mat_stream_kernel<ICONV_MAT_T, false, 1>;
}

}  // namespace

// With programmatic stream serialisation (see grid_dep_wait) and clusters of a pair or of the split.
cudaError_t ICONV_CAT(mat_launch_, ICONV_MAT_ID)(bool gated, const MatLaunch &l)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(l.grid);
    cfg.blockDim = dim3(l.threads);
    cfg.dynamicSmemBytes = l.smem;
    cfg.stream = l.stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = l.bulk ? 2u : (unsigned)l.a->split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    if (l.streams) {
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, stream_instance(gated, l.a->m > 8), *l.s, *l.a);
    }
    cfg.numAttrs = attr[1].val.clusterDim.x == 1 ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, instance(gated, l.bulk), *l.tmap_w, *l.tmap_x, *l.a);
}

cudaError_t ICONV_CAT(mat_opt_in_, ICONV_MAT_ID)()
{
    for (bool gated : {false, true}) {
        for (MatKernel k : {instance(gated, true), instance(gated, false)}) {
            const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM);
            if (e != cudaSuccess) return e;
        }
        for (bool wide : {false, true}) {
            const cudaError_t e = cudaFuncSetAttribute(stream_instance(gated, wide), cudaFuncAttributeMaxDynamicSharedMemorySize, MAT_STREAM_SMEM);
            if (e != cudaSuccess) return e;
        }
    }
    return cudaSuccess;
}

}  // namespace iconv
