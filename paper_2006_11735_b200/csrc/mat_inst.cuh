// Body of one translation unit of product kernels: define ICONV_MAT_T (output type) and ICONV_MAT_ID before including.
#include "mat_inst.h"

namespace iconv {

#define ICONV_CAT2(a, b) a##b
#define ICONV_CAT(a, b) ICONV_CAT2(a, b)

namespace {

using MatKernel = void (*)(CUtensorMap, CUtensorMap, MatArgs);

template <bool GATED>
MatKernel instance(int split)
{
    switch (split) {
    case 0: return mat_bulk_kernel<ICONV_MAT_T, GATED>;
    case 1: return mat_few_kernel<ICONV_MAT_T, GATED, 1>;
    case 2: return mat_few_kernel<ICONV_MAT_T, GATED, 2>;
    case 4: return mat_few_kernel<ICONV_MAT_T, GATED, 4>;
    default: return mat_few_kernel<ICONV_MAT_T, GATED, 8>;
    }
}

}  // namespace

// With programmatic stream serialisation (see grid_dep_wait) and clusters of a pair or of the split.
cudaError_t ICONV_CAT(mat_launch_, ICONV_MAT_ID)(bool gated, const MatLaunch &l)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(l.grid);
    cfg.blockDim = dim3(MAT_THREADS);
    cfg.dynamicSmemBytes = l.smem;
    cfg.stream = l.stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = l.split ? (unsigned)l.split : 2u;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = l.split == 1 ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, gated ? instance<true>(l.split) : instance<false>(l.split), *l.tmap_w, *l.tmap_x, *l.a);
}

cudaError_t ICONV_CAT(mat_opt_in_, ICONV_MAT_ID)()
{
    for (int split : {0, 1, 2, 4, 8})
        for (MatKernel k : {instance<false>(split), instance<true>(split)}) {
            const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM);
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

}  // namespace iconv
