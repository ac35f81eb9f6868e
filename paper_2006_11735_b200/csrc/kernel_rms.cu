// Residual addition, root-mean-square norm and 8-bit rows with a scale each (irms_quant).
//
//   s = x + r,  v = s * g,  a = max|v|,  q = floor(v * (127 / a) + 1/2),  scale = a / 127 * rsqrt(mean(s^2) + eps)
//
// The root cancels in q, so one pass over the row gives everything that the rounding needs (the maximum) and everything that the scale
// needs (the sum of squares), and nothing is read twice: a row stays in its threads' registers between the two.  The products and sums
// before the rounding are single IEEE operations (no contraction), so q is a function of the row alone, whatever the launch shape.
//
// What bounds it: HBM -- 7 bytes an element with a residual in 16 bits.  One block per row (a warp per row for short ones), vectors of
// 16 bytes per thread.
#include <cfloat>
#include <cstdint>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "plan.h"

namespace iconv {

namespace {

struct RmsArgs {
    const void *x, *r, *g;
    void *sum;
    int8_t *q;
    float *scales;
    long long rows, ldx, ldr, lds, ldq;
    int width, g_f32, norm;
    float eps, inv_width;
};

constexpr int ROW_WARPS_MAX = 32;
constexpr float TINY_ROW = 1.504632769052528e-36f;  // 2^-119: 127 / a is finite from here on
constexpr float DOWN = 7.888609052210118e-31f;      // 2^-100

template <typename T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float to(float v) { return v; }
    static __device__ __forceinline__ float from(float v) { return v; }
};
template <> struct Elem<__half> {
    static __device__ __forceinline__ float to(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half from(float v) { return __float2half_rn(v); }
};
template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float to(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 from(float v) { return __float2bfloat16_rn(v); }
};

// the larger of the two, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// VE elements as they lie in memory: 16 bytes, or a single element
template <typename T, int VE> struct Raw { uint4 w; };
template <typename T> struct Raw<T, 1> { T w; };

template <typename T, int VE>
__device__ __forceinline__ Raw<T, VE> load_raw(const T *p)
{
    Raw<T, VE> v;
    if constexpr (VE > 1) v.w = ld_tensor((const uint4 *)p);
    else v.w = *p;
    return v;
}
template <typename T, int VE>
__device__ __forceinline__ void to_float(const Raw<T, VE> &v, float (&f)[VE])
{
    const T *e = (const T *)&v.w;
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = Elem<T>::to(e[j]);
}
template <typename T, int VE>
__device__ __forceinline__ void store_elems(T *p, const float (&f)[VE])
{
    Raw<T, VE> v;
    T *e = (T *)&v.w;
#pragma unroll
    for (int j = 0; j < VE; ++j) e[j] = Elem<T>::from(f[j]);
    if constexpr (VE > 1) *(uint4 *)p = v.w;
    else *p = v.w;
}
// floor(v * inv + 1/2); the sum is rounded down, so that a value just under the border stays under it.  NaN gives 0.
__device__ __forceinline__ int round_q(float v, float inv) { return __float2int_rd(__fadd_rd(__fmul_rn(v, inv), 0.5f)); }

template <int VE>
__device__ __forceinline__ void store_q(int8_t *p, const float (&v)[VE], float inv)
{
    unsigned b[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) b[j] = (unsigned)round_q(v[j], inv);
    if constexpr (VE > 1) {
#pragma unroll
        for (int w = 0; w < VE / 4; ++w) b[w] = __byte_perm(__byte_perm(b[4 * w], b[4 * w + 1], 0x0040), __byte_perm(b[4 * w + 2], b[4 * w + 3], 0x0040), 0x5410);
        if constexpr (VE == 8) *(uint2 *)p = make_uint2(b[0], b[1]);
        else *(unsigned *)p = b[0];
    } else {
        *p = (int8_t)b[0];
    }
}

// What a row's threads gather: the sum of squares, the same of the values 2^-100 of themselves (finite where the other is not), the largest magnitude.
struct RowSums {
    float sq, sq_down, top;
    __device__ __forceinline__ void join(const RowSums &o)
    {
        sq += o.sq;
        sq_down += o.sq_down;
        top = max_nan(top, o.top);
    }
};

// Over the TPR threads of a row (a warp's, or the whole block's); every thread gets the result.
template <int TPR>
__device__ __forceinline__ void row_reduce(RowSums &m, RowSums *sh)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        m.join({__shfl_xor_sync(0xffffffffu, m.sq, o), __shfl_xor_sync(0xffffffffu, m.sq_down, o), __shfl_xor_sync(0xffffffffu, m.top, o)});
    if (TPR > 32) {
        if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = m;
        __syncthreads();
        m = sh[0];
#pragma unroll
        for (int w = 1; w < TPR / 32; ++w) m.join(sh[w]);
    }
}

// TPR threads a row, R vectors of VE elements each in registers (R = 0: any width, the row is read twice).
template <typename T, int VE, int TPR, int R>
__global__ void __launch_bounds__(TPR > 128 ? TPR : 128) rms_quant_kernel(const __grid_constant__ RmsArgs a)
{
    constexpr int ROWS = TPR > 128 ? 1 : 128 / TPR;
    constexpr int HELD = R > 0 ? R : 1;
    static_assert(ROWS == 1 || TPR == 32, "several rows a block: a warp each");
    __shared__ RowSums sh[ROW_WARPS_MAX];
    grid_dep_launch();
    grid_dep_wait();
    const int t = ROWS > 1 ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
    const long long row = (long long)blockIdx.x * ROWS + (ROWS > 1 ? (int)(threadIdx.x >> 5) : 0);
    if (row >= a.rows) return;
    const T *x = (const T *)a.x + row * a.ldx;
    const T *r = a.r ? (const T *)a.r + row * a.ldr : nullptr;
    T *out = a.sum ? (T *)a.sum + row * a.lds : nullptr;
    int8_t *q = a.q + row * a.ldq;
    const int vecs = a.width / VE;
    RowSums m = {0.0f, 0.0f, 0.0f};

    // s of a vector, from what was loaded of x and the residual
    auto add = [&](const Raw<T, VE> &xr, const Raw<T, VE> &rr, float (&s)[VE]) {
        to_float<T, VE>(xr, s);
        if (r) {
            float o[VE];
            to_float<T, VE>(rr, o);
#pragma unroll
            for (int j = 0; j < VE; ++j) s[j] = __fadd_rn(s[j], o[j]);
        }
    };
    auto weigh = [&](int i, const Raw<T, VE> &gr, float (&s)[VE]) {
        if (a.g && a.g_f32) {
#pragma unroll
            for (int j = 0; j < VE; ++j) s[j] = __fmul_rn(s[j], ((const float *)a.g)[i * VE + j]);
        } else if (a.g) {
            float g[VE];
            to_float<T, VE>(gr, g);
#pragma unroll
            for (int j = 0; j < VE; ++j) s[j] = __fmul_rn(s[j], g[j]);
        }
    };
    auto squares = [&](const float (&s)[VE]) {
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            m.sq = fmaf(s[j], s[j], m.sq);
            if (!std::is_same<T, __half>::value) m.sq_down = fmaf(s[j] * DOWN, s[j] * DOWN, m.sq_down);      // (no sum of two halves needs it)
        }
    };
    auto largest = [&](const float (&v)[VE]) {
#pragma unroll
        for (int j = 0; j < VE; ++j) m.top = max_nan(m.top, fabsf(v[j]));
    };
    // vector i of x, the residual and the weight; each load is issued whether or not the thread has such a vector (it then reads the
    // last one), so that none waits behind a branch for the one before it
    auto fetch = [&](int i, Raw<T, VE> &xr, Raw<T, VE> &rr, Raw<T, VE> &gr) {
        const int at = (i < vecs ? i : vecs - 1) * VE;
        xr = load_raw<T, VE>(x + at);
        if (r) rr = load_raw<T, VE>(r + at);
        if (a.g && !a.g_f32) gr = load_raw<T, VE>((const T *)a.g + at);
    };

    float v[HELD][VE];
    if (R > 0) {
        Raw<T, VE> xr[HELD], rr[HELD], gr[HELD];
#pragma unroll
        for (int i = 0; i < R; ++i) fetch(i * TPR + t, xr[i], rr[i], gr[i]);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int at = i * TPR + t;
            if (at < vecs) {
                add(xr[i], rr[i], v[i]);
                if (out) store_elems<T, VE>(out + at * VE, v[i]);
                squares(v[i]);
                weigh(at, gr[i], v[i]);
                largest(v[i]);
            }
        }
    } else {
        for (int at = t; at < vecs; at += TPR) {
            Raw<T, VE> xr, rr, gr;
            fetch(at, xr, rr, gr);
            add(xr, rr, v[0]);
            squares(v[0]);
            weigh(at, gr, v[0]);
            largest(v[0]);
        }
    }
    row_reduce<TPR>(m, sh);

    const bool broken = !(m.top <= FLT_MAX);                       // a NaN or an infinity in the row
    const bool empty = m.top < TINY_ROW;
    float scale = m.top * (1.0f / 127.0f);
    if (a.norm) {
        // (where the squares of finite values do not fit, eps is nothing beside them)
        if (m.sq <= FLT_MAX) scale *= 1.0f / sqrtf(fmaf(m.sq, a.inv_width, a.eps));
        else scale = scale * DOWN / sqrtf(m.sq_down * a.inv_width);
    }
    const float inv = broken || empty ? 0.0f : __fdiv_rn(127.0f, m.top);
    if (t == 0) a.scales[row] = broken ? __int_as_float(0x7fffffff) : empty ? 0.0f : scale;

    if (R > 0) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int at = i * TPR + t;
            if (at < vecs) store_q<VE>(q + at * VE, v[i], inv);
        }
    } else {
        for (int at = t; at < vecs; at += TPR) {
            Raw<T, VE> xr, rr, gr;
            fetch(at, xr, rr, gr);
            add(xr, rr, v[0]);
            if (out) store_elems<T, VE>(out + at * VE, v[0]);       // (only now: it may be where x or the residual is)
            weigh(at, gr, v[0]);
            store_q<VE>(q + at * VE, v[0], inv);
        }
    }
}

template <typename T, int VE, int TPR, int R>
cudaError_t launch_one(const RmsArgs &a, cudaStream_t stream)
{
    constexpr int ROWS = TPR > 128 ? 1 : 128 / TPR;
    const long long blocks = (a.rows + ROWS - 1) / ROWS;
    const auto kernel = rms_quant_kernel<T, VE, TPR, R>;
    return launch_kernel(kernel, true, (unsigned)blocks, TPR > 128 ? TPR : 128, 0, stream, a);
}

template <typename T, int VE>
cudaError_t launch_width(const RmsArgs &a, cudaStream_t stream)
{
    const int vecs = a.width / VE;
    if constexpr (VE > 1) {
        if (vecs <= 32) return launch_one<T, VE, 32, 1>(a, stream);
        if (vecs <= 64) return launch_one<T, VE, 32, 2>(a, stream);
        if (vecs <= 128) return launch_one<T, VE, 128, 1>(a, stream);
        if (vecs <= 256) return launch_one<T, VE, 128, 2>(a, stream);
        if (vecs <= 512) return launch_one<T, VE, 256, 2>(a, stream);
        if (vecs <= 1024) return launch_one<T, VE, 512, 2>(a, stream);
        if (vecs <= 2048) return launch_one<T, VE, 512, 4>(a, stream);
        if (vecs <= 4096) return launch_one<T, VE, 1024, 4>(a, stream);
        return launch_one<T, VE, 1024, 0>(a, stream);
    } else {
        if (vecs <= 128) return launch_one<T, VE, 32, 4>(a, stream);
        if (vecs <= 1024) return launch_one<T, VE, 128, 8>(a, stream);
        if (vecs <= 4096) return launch_one<T, VE, 256, 16>(a, stream);
        if (vecs <= 16384) return launch_one<T, VE, 1024, 16>(a, stream);
        return launch_one<T, VE, 1024, 0>(a, stream);
    }
}

template <typename T>
int launch_rms(const RmsArgs &a, bool whole, cudaStream_t stream)
{
    constexpr int VE = 16 / (int)sizeof(T);
    ICONV_CUDA_TRY((whole ? launch_width<T, VE>(a, stream) : launch_width<T, 1>(a, stream)));
    return ICONV_OK;
}

int size_of(int dtype) { return dtype == ICONV_F32 ? 4 : 2; }

}  // namespace

}  // namespace iconv

using namespace iconv;

extern "C" int irms_quant(const irms_desc *desc, const void *x, const void *residual, const void *weight, void *sum, int8_t *q, float *scales,
                          void *cuda_stream)
{
    if (!desc) { set_error("irms_quant: null descriptor"); return ICONV_ERR_ARG; }
    const irms_desc &d = *desc;
    if (d.rows < 0 || d.width < 1) { set_error("irms_quant: need rows >= 0 and width >= 1"); return ICONV_ERR_ARG; }
    if (d.dtype != ICONV_F32 && d.dtype != ICONV_F16 && d.dtype != ICONV_BF16) { set_error("irms_quant: dtype must be F32, F16 or BF16"); return ICONV_ERR_ARG; }
    if (weight && d.weight_dtype != d.dtype && d.weight_dtype != ICONV_F32) { set_error("irms_quant: weight_dtype must be dtype or F32"); return ICONV_ERR_ARG; }
    if (!(d.eps >= 0.0f) || d.eps > 3.4028235e38f) { set_error("irms_quant: eps must be finite and not negative"); return ICONV_ERR_ARG; }
    if (d.norm != 0 && d.norm != 1) { set_error("irms_quant: norm must be 0 or 1"); return ICONV_ERR_ARG; }
    if (d.x_stride < d.width || d.q_stride < d.width || (residual && d.residual_stride < d.width) || (sum && d.sum_stride < d.width)) {
        set_error("irms_quant: a row stride is shorter than the row");
        return ICONV_ERR_SHAPE;
    }
    if (d.rows > 0x7fffffffll) { set_error("irms_quant: at most 2^31 - 1 rows"); return ICONV_ERR_SHAPE; }
    const long long most = 1ll << 46;                               // elements from a matrix's first row to its last
    if (d.rows > 0 && (d.x_stride > most / d.rows || d.q_stride > most / d.rows || (residual && d.residual_stride > most / d.rows) ||
                       (sum && d.sum_stride > most / d.rows))) {
        set_error("irms_quant: matrix too large");
        return ICONV_ERR_SHAPE;
    }
    if (d.rows == 0) return ICONV_OK;
    if (!x || !q || !scales) { set_error("irms_quant: x, q and scales must be given"); return ICONV_ERR_ARG; }
    const int e = size_of(d.dtype);
    if (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)sum) % e || (weight && (uintptr_t)weight % size_of(d.weight_dtype)) || (uintptr_t)scales % 4) {
        set_error("irms_quant: an address is not aligned to its element");
        return ICONV_ERR_ALIGN;
    }
    RmsArgs a;
    a.x = x; a.r = residual; a.g = weight; a.sum = sum; a.q = q; a.scales = scales;
    a.rows = d.rows; a.ldx = d.x_stride; a.ldr = d.residual_stride; a.lds = d.sum_stride; a.ldq = d.q_stride;
    a.width = d.width; a.g_f32 = d.weight_dtype == ICONV_F32; a.norm = d.norm; a.eps = d.eps; a.inv_width = 1.0f / (float)d.width;
    const int ve = 16 / e;                                          // elements of a vector; the same number of bytes of q
    bool whole = !(d.width % ve) && !(((uintptr_t)x | (uintptr_t)residual | (uintptr_t)sum) % 16) && !((uintptr_t)q % ve) && !(d.x_stride % ve) && !(d.q_stride % ve);
    if (residual) whole = whole && !(d.residual_stride % ve);
    if (sum) whole = whole && !(d.sum_stride % ve);
    if (weight && !(a.g_f32 && d.dtype != ICONV_F32)) whole = whole && !((uintptr_t)weight % 16);
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (d.dtype == ICONV_F32) { a.g_f32 = 0; return launch_rms<float>(a, whole, stream); }
    if (d.dtype == ICONV_F16) return launch_rms<__half>(a, whole, stream);
    return launch_rms<__nv_bfloat16>(a, whole, stream);
}
