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
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "umma_device.cuh"

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
constexpr float UP = 1.2379400392853803e+27f;       // 2^90
constexpr float MUCH = 1.0e25f, LITTLE = 1.0e-18f;  // sums of squares beyond which others are kept besides

template <typename T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float to(float v) { return v; }
    static __device__ __forceinline__ float from(float v) { return v; }
};
template <> struct Elem<__half> {
    static __device__ __forceinline__ float to(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half from(float v) { return __float2half_rn(v); }
    using Two = __half2;
    static __device__ __forceinline__ Two from2(float a, float b) { return __floats2half2_rn(a, b); }
};
template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float to(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 from(float v) { return __float2bfloat16_rn(v); }
    using Two = __nv_bfloat162;
    static __device__ __forceinline__ Two from2(float a, float b) { return __floats2bfloat162_rn(a, b); }
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
    if constexpr (VE == 8) {
        using Two = typename Elem<T>::Two;
        union { Two t[4]; uint4 w; } v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v.t[j] = Elem<T>::from2(f[2 * j], f[2 * j + 1]);
        *(uint4 *)p = v.w;
    } else if constexpr (VE == 4) {
        *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
    } else {
        *p = Elem<T>::from(f[0]);
    }
}
// floor(v * inv + 1/2) in the low byte: both sums are rounded down, the first so that a value just under the border stays under it, the second
// leaves the whole number beside 1.5 * 2^23 (an addition where a conversion runs at an eighth of the rate).  For |v * inv| of 127 and a rounding.
__device__ __forceinline__ unsigned round_q(float v, float inv) { return __float_as_uint(__fadd_rd(__fadd_rd(__fmul_rn(v, inv), 0.5f), 12582912.0f)); }
// ... of two values at a time: the same operations, two in an instruction
__device__ __forceinline__ unsigned long long two(float a, float b)
{
    unsigned long long d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ void round_q2(float a, float b, unsigned long long inv, unsigned &qa, unsigned &qb)
{
    unsigned long long t;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(t) : "l"(two(a, b)), "l"(inv));
    asm("add.rm.f32x2 %0, %0, %1;" : "+l"(t) : "l"(two(0.5f, 0.5f)));
    asm("add.rm.f32x2 %0, %0, %1;" : "+l"(t) : "l"(two(12582912.0f, 12582912.0f)));
    asm("mov.b64 {%0, %1}, %2;" : "=r"(qa), "=r"(qb) : "l"(t));
}

// inv = 0 (nothing in the row, or something that is no number): zeros
template <int VE>
__device__ __forceinline__ void store_q(int8_t *p, const float (&v)[VE], float inv)
{
    unsigned b[VE];
    if constexpr (VE > 1) {
#pragma unroll
        for (int j = 0; j < VE; j += 2) round_q2(v[j], v[j + 1], two(inv, inv), b[j], b[j + 1]);
#pragma unroll
        for (int w = 0; w < VE / 4; ++w) {
            b[w] = __byte_perm(__byte_perm(b[4 * w], b[4 * w + 1], 0x0040), __byte_perm(b[4 * w + 2], b[4 * w + 3], 0x0040), 0x5410);
            if (inv == 0.0f) b[w] = 0;
        }
        if constexpr (VE == 8) *(uint2 *)p = make_uint2(b[0], b[1]);
        else *(unsigned *)p = b[0];
    } else {
        b[0] = round_q(v[0], inv);
        *p = inv == 0.0f ? (int8_t)0 : (int8_t)b[0];
    }
}

// What a row's threads gather: the sum of squares and the largest magnitude.
struct RowSums {
    float sq, top;
    template <int VE>
    __device__ __forceinline__ void largest(const float (&v)[VE])
    {
#pragma unroll
        for (int j = 0; j < VE; ++j) top = max_nan(top, fabsf(v[j]));
    }
    __device__ __forceinline__ void join(const RowSums &o)
    {
        sq += o.sq;
        top = max_nan(top, o.top);
    }
};

// The far sum, for a row whose sum of squares is too large or too small for a float: of the values 2^-100 of themselves where a thread's
// squares pass MUCH (what other threads hold is nothing beside a sum that does not fit), or, as a negative number, of the values 2^90 of themselves where
// they stay under LITTLE and eps does not cover them.
template <int R, int VE>
__device__ __forceinline__ void add_far(const float (&s)[R][VE], bool much, float &far)
{
    const float by = much ? DOWN : UP;
    float f = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j) f = fmaf(s[i][j] * by, s[i][j] * by, f);
    far += much ? f : -f;
}
// Squares of a thread's whole share of a row.
template <int R, int VE>
__device__ __forceinline__ float squares(const float (&s)[R][VE])
{
    if constexpr (VE > 1) {
        unsigned long long t = 0;
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < VE; j += 2) {
                const unsigned long long e = two(s[i][j], s[i][j + 1]);
                asm("fma.rn.f32x2 %0, %1, %1, %0;" : "+l"(t) : "l"(e));
            }
        float lo, hi;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(t));
        return lo + hi;
    } else {
        float p = 0.0f;
#pragma unroll
        for (int i = 0; i < R; ++i) p = fmaf(s[i][0], s[i][0], p);
        return p;
    }
}
// ... and the far sum with it, where s is gone when the row's sum is known
template <int R, int VE>
__device__ __forceinline__ float squares_and_far(const float (&s)[R][VE], float eps, float &far)
{
    const float p = squares(s);
    if (p > MUCH || (eps < LITTLE && p < LITTLE)) add_far(s, p > MUCH, far);
    return p;
}
// Whether the far sums decide, and a thread's part of them.
__device__ __forceinline__ bool far_decides(const RmsArgs &a, const RowSums &m) { return a.norm && (!(m.sq <= FLT_MAX) || (m.sq < LITTLE && a.eps < LITTLE)); }
__device__ __forceinline__ float far_part(const RowSums &m, float far) { return m.sq < LITTLE ? -far : fmaxf(far, 0.0f); }

// Over the TPR threads of a row (a warp's, or the whole block's); every thread gets the result.
template <int TPR>
__device__ __forceinline__ void row_reduce(RowSums &m, RowSums *sh)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m.join({__shfl_xor_sync(0xffffffffu, m.sq, o), __shfl_xor_sync(0xffffffffu, m.top, o)});
    if (TPR > 32) {
        if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = m;
        __syncthreads();
        m = sh[0];
#pragma unroll
        for (int w = 1; w < TPR / 32; ++w) m.join(sh[w]);
    }
}
template <int TPR>
__device__ __forceinline__ float far_reduce(float f, RowSums *sh)
{
#pragma unroll 1
    for (int o = 16; o > 0; o >>= 1) f += __shfl_xor_sync(0xffffffffu, f, o);
    if (TPR > 32) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5].sq = f;
        __syncthreads();
        f = 0.0f;
#pragma unroll 1
        for (int w = 0; w < TPR / 32; ++w) f += sh[w].sq;
    }
    return f;
}

// The row's scale (stored by `stores`), and what v is multiplied by before it is rounded.  far: of the whole row, where it decides.
__device__ __forceinline__ float finish_row(const RmsArgs &a, const RowSums &m, float far, long long row, bool stores)
{
    const bool broken = !(m.top <= FLT_MAX);                       // a NaN or an infinity in the row
    const bool empty = m.top < TINY_ROW;
    float scale = m.top * (1.0f / 127.0f);
    if (!far_decides(a, m)) {
        if (a.norm) scale *= 0.5f * (1.0f / sqrtf(fmaf(0.25f * m.sq, a.inv_width, 0.25f * a.eps)));       // (their sum may not fit either)
    } else if (m.sq < LITTLE) {
        const float root = sqrtf(fmaf(far, a.inv_width, a.eps * UP * UP));
        scale = scale < 1.0f ? scale * UP / root : scale / root * UP;
    } else {
        scale /= fminf(sqrtf(fmaf(far, a.inv_width, a.eps * DOWN * DOWN)) * (1.0f / DOWN), FLT_MAX);     // (the root itself is a float)
    }
    if (stores) a.scales[row] = broken ? __int_as_float(0x7fffffff) : empty ? 0.0f : scale;
    return broken || empty ? 0.0f : __fdiv_rn(127.0f, m.top);
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
    RowSums m = {0.0f, 0.0f};
    float far = 0.0f;

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
    // vector i of x, the residual and the weight; each load is issued whether or not the thread has such a vector (it then reads the
    // last one), so that none waits behind a branch for the one before it
    auto fetch = [&](int i, Raw<T, VE> &xr, Raw<T, VE> &rr, Raw<T, VE> &gr) {
        const int at = (i < vecs ? i : vecs - 1) * VE;
        xr = load_raw<T, VE>(x + at);
        if (r) rr = load_raw<T, VE>(r + at);
        if (a.g && !a.g_f32) gr = load_raw<T, VE>((const T *)a.g + at);
    };

    // float rows, and rows that are not held, are read again in the rare case that the far sum decides; others keep it from the start
    constexpr bool AGAIN = R == 0 || sizeof(T) == 4;
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
                if constexpr (VE == 1 && AGAIN) {   // (single elements: one loop costs less than two)
                    m.sq = fmaf(v[i][0], v[i][0], m.sq);
                    weigh(at, gr[i], v[i]);
                    m.largest(v[i]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < VE; ++j) v[i][j] = 0.0f;
            }
        }
        if constexpr (VE > 1 || !AGAIN) {
            if (a.norm) m.sq = AGAIN ? squares(v) : squares_and_far(v, a.eps, far);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int at = i * TPR + t;
                if (at < vecs) {
                    weigh(at, gr[i], v[i]);
                    m.largest(v[i]);
                }
            }
        }
    } else {
        for (int at = t; at < vecs; at += TPR) {
            Raw<T, VE> xr, rr, gr;
            fetch(at, xr, rr, gr);
            add(xr, rr, v[0]);
            m.sq += squares(v);
            weigh(at, gr, v[0]);
            m.largest(v[0]);
        }
    }
    row_reduce<TPR>(m, sh);

    if (far_decides(a, m)) {
        if constexpr (AGAIN)
#pragma unroll 1
            for (int at = t; at < vecs; at += TPR) {
                Raw<T, VE> xr, rr, gr;
                float s[1][VE];
                fetch(at, xr, rr, gr);
                if (R > 0 && out) to_float<T, VE>(load_raw<T, VE>(out + at * VE), s[0]);       // (it may be where x or the residual was; float: as it is)
                else add(xr, rr, s[0]);
                add_far(s, !(m.sq < LITTLE), far);
            }
        far = far_reduce<TPR>(far_part(m, far), sh);
    }
    const float inv = finish_row(a, m, far, row, t == 0);

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

// ---- Rows of 16-bit elements that start anywhere (an odd width without padding): vectors of 16 bytes all the same (2000 rows of 16001 with a
// residual: 86 us, 367 element by element, floor 34; 8192 of 4001 alone 46 and 80, floor 15; in float single elements are as fast: 4000 of 1501 18 us, 20 so, 2000 of 8191 54 and 54).  A thread's VE
// elements lie across two aligned 16-byte words; both are loaded (the second is the neighbour's first, and in L1) and shifted by the row's phase,
// which is the same for all its threads.  The sum goes back the other way: a lane stores the aligned word that its own elements and the
// lane's before it make up, and the ends of a warp's stretch go out element by element.  q's rows are aligned.
// 1024 threads of 64 registers on an SM, at the price of a word or two of spills (82 registers: 2000 rows of 8191 with a residual 58 us, 40 so).

// Bytes off ... off + 15 of the 32 that a and b make.
__device__ __forceinline__ uint4 cut16(const uint4 &a, const uint4 &b, unsigned off)
{
    const unsigned bits = (off & 3u) * 8u;
    uint4 d;
    switch (off >> 2) {
    case 0:
        d.x = __funnelshift_r(a.x, a.y, bits); d.y = __funnelshift_r(a.y, a.z, bits); d.z = __funnelshift_r(a.z, a.w, bits); d.w = __funnelshift_r(a.w, b.x, bits);
        break;
    case 1:
        d.x = __funnelshift_r(a.y, a.z, bits); d.y = __funnelshift_r(a.z, a.w, bits); d.z = __funnelshift_r(a.w, b.x, bits); d.w = __funnelshift_r(b.x, b.y, bits);
        break;
    case 2:
        d.x = __funnelshift_r(a.z, a.w, bits); d.y = __funnelshift_r(a.w, b.x, bits); d.z = __funnelshift_r(b.x, b.y, bits); d.w = __funnelshift_r(b.y, b.z, bits);
        break;
    default:
        d.x = __funnelshift_r(a.w, b.x, bits); d.y = __funnelshift_r(b.x, b.y, bits); d.z = __funnelshift_r(b.y, b.z, bits); d.w = __funnelshift_r(b.z, b.w, bits);
        break;
    }
    return d;
}

// A matrix to be read so: its first and last 16-byte words that lie in it whole.
struct Window {
    const char *first, *last;
};
// The two words around a vector; near the matrix's ends other ones of it instead (exact: those were the right ones).
struct Pair {
    uint4 a, b;
    bool exact;
};
__device__ __forceinline__ Pair load_pair(const char *at, const Window &w)
{
    const char *base = at - ((uintptr_t)at & 15);
    const char *from = base < w.first ? w.first : base + 16 > w.last ? w.last - 16 : base;
    Pair p;
    p.a = ld_tensor((const uint4 *)from);
    p.b = ld_tensor((const uint4 *)from + 1);
    p.exact = from == base;
    return p;
}
// ... as numbers; `count` of them are the row's
template <typename T, int VE>
__device__ __forceinline__ void pair_to_float(const Pair &p, const char *at, int count, float (&f)[VE])
{
    if (p.exact) {
        Raw<T, VE> v;
        v.w = cut16(p.a, p.b, (unsigned)(uintptr_t)at & 15u);
        to_float<T, VE>(v, f);
    } else {
#pragma unroll
        for (int j = 0; j < VE; ++j) f[j] = j < count ? Elem<T>::to(((const T *)at)[j]) : 0.0f;
    }
    if (count < VE)
#pragma unroll
        for (int j = 0; j < VE; ++j) f[j] = j < count ? f[j] : 0.0f;
}
// A warp's vectors to consecutive places from its first lane's `at` on; all lanes take part.  count: this lane's elements (VE, fewer in the row's last
// vector, or none).
template <typename T, int VE>
__device__ __forceinline__ void store_shifted(T *at, const float (&f)[VE], int count, int lane)
{
    union { T e[VE]; uint4 w; } o;
#pragma unroll
    for (int j = 0; j < VE; ++j) o.e[j] = Elem<T>::from(f[j]);
    const unsigned off = (unsigned)(uintptr_t)at & 15u;                      // the same in every lane
    const unsigned whole = __ballot_sync(0xffffffffu, count == VE);          // the first lanes
    int from = 0, to = 0;                                                    // elements that go out one by one
    if (off == 0) {
        if (count == VE) *(uint4 *)at = o.w;
    } else {
        uint4 before;
        before.x = __shfl_up_sync(0xffffffffu, o.w.x, 1); before.y = __shfl_up_sync(0xffffffffu, o.w.y, 1);
        before.z = __shfl_up_sync(0xffffffffu, o.w.z, 1); before.w = __shfl_up_sync(0xffffffffu, o.w.w, 1);
        if (count == VE && lane > 0) *(uint4 *)((char *)at - off) = cut16(before, o.w, 16u - off);
        if (count == VE && lane == 0) to = VE - (int)(off / sizeof(T));
        if (lane == __popc(whole) - 1) {                                     // what the lane behind would have taken along
            if (lane > 0) from = VE - (int)(off / sizeof(T));
            to = VE;
        }
    }
    if (count < VE) to = count;
    if (to > from)
#pragma unroll
        for (int j = 0; j < VE; ++j)
            if (j >= from && j < to) at[j] = o.e[j];
}

struct ShiftArgs {
    RmsArgs a;
    Window x, r, g;
};

template <typename T, int TPR, int R>
__global__ void __launch_bounds__(TPR > 128 ? TPR : 128, TPR == 1024 ? 1 : TPR >= 256 ? 1024 / TPR : 8) rms_shift_kernel(const __grid_constant__ ShiftArgs s)
{
    constexpr int VE = 16 / (int)sizeof(T), ROWS = TPR > 128 ? 1 : 128 / TPR;
    __shared__ RowSums sh[ROW_WARPS_MAX];
    const RmsArgs &a = s.a;
    grid_dep_launch();
    grid_dep_wait();
    const int lane = threadIdx.x & 31, t = ROWS > 1 ? lane : (int)threadIdx.x;
    const long long row = (long long)blockIdx.x * ROWS + (ROWS > 1 ? (int)(threadIdx.x >> 5) : 0);
    if (row >= a.rows) return;
    const char *x = (const char *)((const T *)a.x + row * a.ldx), *r = a.r ? (const char *)((const T *)a.r + row * a.ldr) : nullptr;
    T *out = a.sum ? (T *)a.sum + row * a.lds : nullptr;
    int8_t *q = a.q + row * a.ldq;
    const bool g_pairs = a.g && !a.g_f32;
    RowSums m = {0.0f, 0.0f};
    float far = 0.0f;
    float v[R][VE];
    Pair xp[R], rp[R], gp[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int byte = (i * TPR + t) * 16;
        xp[i] = load_pair(x + byte, s.x);
        if (r) rp[i] = load_pair(r + byte, s.r);
        if (g_pairs) gp[i] = load_pair((const char *)a.g + byte, s.g);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int at = (i * TPR + t) * VE, left = a.width - at, count = left < 0 ? 0 : left < VE ? left : VE;
        pair_to_float<T, VE>(xp[i], x + at * (int)sizeof(T), count, v[i]);
        if (r) {
            float o[VE];
            pair_to_float<T, VE>(rp[i], r + at * (int)sizeof(T), count, o);
#pragma unroll
            for (int j = 0; j < VE; ++j) v[i][j] = __fadd_rn(v[i][j], o[j]);
        }
        if (out) store_shifted<T, VE>(out + at, v[i], count, lane);
    }
    if (a.norm) m.sq = squares_and_far(v, a.eps, far);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int at = (i * TPR + t) * VE, left = a.width - at, count = left < 0 ? 0 : left < VE ? left : VE;
        if (g_pairs) {
            float g[VE];
            pair_to_float<T, VE>(gp[i], (const char *)((const T *)a.g + at), count, g);
#pragma unroll
            for (int j = 0; j < VE; ++j) v[i][j] = __fmul_rn(v[i][j], g[j]);
        } else if (a.g) {
#pragma unroll
            for (int j = 0; j < VE; ++j) v[i][j] = j < count ? __fmul_rn(v[i][j], ((const float *)a.g)[at + j]) : 0.0f;
        }
        m.largest(v[i]);
    }
    row_reduce<TPR>(m, sh);
    if (far_decides(a, m)) far = far_reduce<TPR>(far_part(m, far), sh);
    const float inv = finish_row(a, m, far, row, t == 0);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int at = (i * TPR + t) * VE, count = a.width - at;
        if (count >= VE) {
            store_q<VE>(q + at, v[i], inv);
        } else {
#pragma unroll
            for (int j = 0; j < VE; ++j)
                if (j < count) q[at + j] = inv == 0.0f ? (int8_t)0 : (int8_t)round_q(v[i][j], inv);
        }
    }
}

template <typename T, int TPR, int R>
cudaError_t launch_shift_one(const ShiftArgs &s, cudaStream_t stream)
{
    constexpr int ROWS = TPR > 128 ? 1 : 128 / TPR;
    const auto kernel = rms_shift_kernel<T, TPR, R>;
    return launch_kernel(kernel, true, (unsigned)((s.a.rows + ROWS - 1) / ROWS), TPR > 128 ? TPR : 128, 0, stream, s);
}
constexpr int SHIFT_VECTORS_MAX = 2048;

// Where a matrix has no two whole words to read there is nothing to gain.
bool window_of(const void *p, long long rows, long long stride, int width, int element, Window &w)
{
    const char *begin = (const char *)p, *end = begin + ((rows - 1) * stride + width) * element;
    w.first = begin + (16 - (uintptr_t)begin % 16) % 16;
    w.last = end - (uintptr_t)end % 16 - 16;
    return w.last >= w.first + 16;
}
template <typename T>
bool shift_args(const RmsArgs &a, ShiftArgs &s)
{
    constexpr int VE = 16 / (int)sizeof(T), E = (int)sizeof(T);
    s.a = a;
    return !((uintptr_t)a.q % VE) && !(a.ldq % VE) && (a.width + VE - 1) / VE <= SHIFT_VECTORS_MAX && window_of(a.x, a.rows, a.ldx, a.width, E, s.x) &&
           (!a.r || window_of(a.r, a.rows, a.ldr, a.width, E, s.r)) && (!a.g || a.g_f32 || window_of(a.g, 1, a.width, a.width, E, s.g));
}
template <typename T>
cudaError_t launch_shift(const ShiftArgs &s, cudaStream_t stream)
{
    const int vecs = (s.a.width + 16 / (int)sizeof(T) - 1) / (16 / (int)sizeof(T));
    if (vecs <= 32) return launch_shift_one<T, 32, 1>(s, stream);
    if (vecs <= 64) return launch_shift_one<T, 32, 2>(s, stream);
    if (vecs <= 128) return launch_shift_one<T, 128, 1>(s, stream);
    if (vecs <= 256) return launch_shift_one<T, 128, 2>(s, stream);
    if (vecs <= 512) return launch_shift_one<T, 256, 2>(s, stream);
    if (vecs <= 1024) return launch_shift_one<T, 512, 2>(s, stream);
    return launch_shift_one<T, 1024, 2>(s, stream);
}

// Many wide rows: one block per SM, whose loading warps keep a ring of whole rows in shared memory ahead of the arithmetic, so that the memory
// stays busy while a row is being reduced (a block per row has nothing in flight then: 4096 rows of 16384 in bfloat16 took 86 us, 41 this
// way, floor 31).  Groups of GW warps take the rows in turn, ELEMS elements a thread; a group meets at one named barrier per row.  The ring's stages
// are a multiple of the groups, so that a stage always holds rows of one group, which has taken the one before when it waits for the next (the
// loads may complete in any order, and a parity cannot tell two rows apart).
constexpr int STREAM_WARPS = 16;                    // that do the arithmetic
constexpr int STREAM_LOADERS = 2;                   // warp 0 loads x, warp 1 the residual
constexpr int STREAM_STAGES_MAX = 16;

struct StreamShared {
    unsigned long long full[STREAM_STAGES_MAX], empty[STREAM_STAGES_MAX];
    RowSums sums[2][STREAM_WARPS];
    volatile int abort_flag;
};

struct StreamArgs {
    RmsArgs a;
    int stages, row_bytes, stage_bytes;             // row_bytes: of x, and of the residual
    int *status;
};

template <typename T, int GW, int ELEMS>
__global__ void __launch_bounds__(32 * (STREAM_WARPS + STREAM_LOADERS), 1) rms_stream_kernel(const __grid_constant__ StreamArgs s)
{
    constexpr int VE = 16 / (int)sizeof(T), R = ELEMS / VE, GROUPS = STREAM_WARPS / GW, TPR = 32 * GW;
    extern __shared__ __align__(16) uint8_t ring[];
    StreamShared *sh = (StreamShared *)(ring + (size_t)s.stages * s.stage_bytes);
    const RmsArgs &a = s.a;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    if (warp == 0) {
        if (lane < s.stages) {
            mbar_init(smem_u32(&sh->full[lane]), a.r ? 2 : 1);
            mbar_init(smem_u32(&sh->empty[lane]), GW);
        }
        if (lane == 0) sh->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    grid_dep_launch();
    grid_dep_wait();
    const long long rows = (a.rows - blockIdx.x + gridDim.x - 1) / gridDim.x;        // of this block: blockIdx.x, + gridDim.x, ...
    auto gave_up = [&](int code) {
        sh->abort_flag = 1;
        atomicCAS(s.status, 0, code);
    };
    if (warp < STREAM_LOADERS) {
        if (lane == 0 && (warp == 0 || a.r)) {
            const char *src = (const char *)(warp == 0 ? a.x : a.r) + (long long)blockIdx.x * (warp == 0 ? a.ldx : a.ldr) * (long long)sizeof(T);
            const long long step = (long long)gridDim.x * (warp == 0 ? a.ldx : a.ldr) * (long long)sizeof(T);
            int stage = 0;
            uint32_t parity = 0;
            for (long long j = 0; j < rows; ++j, src += step) {
                if (!mbar_wait(smem_u32(&sh->empty[stage]), parity ^ 1u, &sh->abort_flag)) { gave_up(1); break; }
                const uint32_t full = smem_u32(&sh->full[stage]);
                mbar_expect_tx(full, (uint32_t)s.row_bytes);
                bulk_load(smem_u32(ring + (size_t)stage * s.stage_bytes + (warp ? s.row_bytes : 0)), src, (uint32_t)s.row_bytes, full);
                if (++stage == s.stages) { stage = 0; parity ^= 1u; }
            }
        }
        __syncwarp();
    } else {
        const int group = (warp - STREAM_LOADERS) / GW, in_group = (warp - STREAM_LOADERS) % GW, t = in_group * 32 + lane;
        const int vecs = a.width / VE;
        constexpr bool HELD = ELEMS <= 32;          // the weights of this thread's elements, the same for every row, stay in registers
        uint4 g[HELD ? R : 1];
        if (HELD && a.g && !a.g_f32)
#pragma unroll
            for (int i = 0; i < R; ++i) g[HELD ? i : 0] = ld_tensor((const uint4 *)((const T *)a.g + (i * TPR + t < vecs ? i * TPR + t : vecs - 1) * VE));
        int stage = group % s.stages, turn = 0;
        uint32_t parity = (uint32_t)(group / s.stages) & 1u;
        // (a wait that runs out leaves its mark and the loop goes on with what there is: every thread meets its group's barrier as often as the others)
        for (long long j = group; j < rows; j += GROUPS, turn ^= 1) {
            const long long row = blockIdx.x + j * gridDim.x;
            if (!mbar_wait(smem_u32(&sh->full[stage]), parity, &sh->abort_flag)) gave_up(2);
            const uint32_t at = smem_u32(ring + (size_t)stage * s.stage_bytes) + (uint32_t)(t * 16);
            T *out = a.sum ? (T *)a.sum + row * a.lds : nullptr;
            RowSums m = {0.0f, 0.0f};
            float far = 0.0f;
            float v[R][VE];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                if (i * TPR + t < vecs) {
                    Raw<T, VE> raw;
                    raw.w = lds128(at + (uint32_t)(i * TPR * 16));
                    to_float<T, VE>(raw, v[i]);
                    if (a.r) {
                        float o[VE];
                        raw.w = lds128(at + (uint32_t)(s.row_bytes + i * TPR * 16));
                        to_float<T, VE>(raw, o);
#pragma unroll
                        for (int e = 0; e < VE; ++e) v[i][e] = __fadd_rn(v[i][e], o[e]);
                    }
                    if (out) store_elems<T, VE>(out + (i * TPR + t) * VE, v[i]);
                } else {
#pragma unroll
                    for (int e = 0; e < VE; ++e) v[i][e] = 0.0f;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->empty[stage]));             // the row is in registers
            if (a.norm) m.sq = squares_and_far(v, a.eps, far);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                if (i * TPR + t < vecs) {
                    if (a.g && a.g_f32) {
#pragma unroll
                        for (int e = 0; e < VE; ++e) v[i][e] = __fmul_rn(v[i][e], ((const float *)a.g)[(i * TPR + t) * VE + e]);
                    } else if (a.g) {
                        Raw<T, VE> raw;
                        float w[VE];
                        raw.w = HELD ? g[HELD ? i : 0] : ld_tensor((const uint4 *)((const T *)a.g + (i * TPR + t) * VE));
                        to_float<T, VE>(raw, w);
#pragma unroll
                        for (int e = 0; e < VE; ++e) v[i][e] = __fmul_rn(v[i][e], w[e]);
                    }
                    m.largest(v[i]);
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m.join({__shfl_xor_sync(0xffffffffu, m.sq, o), __shfl_xor_sync(0xffffffffu, m.top, o)});
            if (lane == 0) sh->sums[turn][warp - STREAM_LOADERS] = m;
            asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(TPR) : "memory");
            m = sh->sums[turn][group * GW];
#pragma unroll
            for (int w = 1; w < GW; ++w) m.join(sh->sums[turn][group * GW + w]);
            if (far_decides(a, m)) {
                far = far_part(m, far);
                for (int o = 16; o > 0; o >>= 1) far += __shfl_xor_sync(0xffffffffu, far, o);
                asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(TPR) : "memory");
                if (lane == 0) sh->sums[turn][warp - STREAM_LOADERS].sq = far;
                asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(TPR) : "memory");
                far = 0.0f;
                for (int w = 0; w < GW; ++w) far += sh->sums[turn][group * GW + w].sq;
            }
            const float inv = finish_row(a, m, far, row, t == 0);
            int8_t *q = a.q + row * a.ldq;
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (i * TPR + t < vecs) store_q<VE>(q + (i * TPR + t) * VE, v[i], inv);
            for (int skip = 0; skip < GROUPS; ++skip)
                if (++stage == s.stages) { stage = 0; parity ^= 1u; }
        }
    }
    __syncthreads();
    if (sh->abort_flag && threadIdx.x == 0) {       // whatever is still on its way into this block's memory
        const long long t0 = clock64();
        while (clock64() - t0 < 4000000) {}
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
        // (instances within a factor of two of the width: what a thread asks for beyond the row's end costs as much as the rest -- 20000
        // float rows of 255 take 13 us with eight elements a lane, 33 with eight in each thread of four warps; 2000 of 5001 47 and, over 1024 threads, 81)
        if (vecs <= 128) return launch_one<T, VE, 32, 4>(a, stream);
        if (vecs <= 256) return launch_one<T, VE, 32, 8>(a, stream);
        if (vecs <= 512) return launch_one<T, VE, 128, 4>(a, stream);
        if (vecs <= 1024) return launch_one<T, VE, 128, 8>(a, stream);
        if (vecs <= 2048) return launch_one<T, VE, 256, 8>(a, stream);
        if (vecs <= 4096) return launch_one<T, VE, 256, 16>(a, stream);
        if (vecs <= 8192) return launch_one<T, VE, 512, 16>(a, stream);
        if (vecs <= 16384) return launch_one<T, VE, 1024, 16>(a, stream);
        return launch_one<T, VE, 1024, 0>(a, stream);
    }
}

using StreamKernel = void (*)(StreamArgs);

// Groups that a block's warps make for rows of a width: eight of two warps, four or two, 32 elements a thread.  The widest rows: one group, unless
// nothing but the row is read (`bare`); then the arithmetic is the bound and two groups of 64 elements a thread take turns (4096 rows of 16384: 41 us,
// 58 in one group; with a residual and weights 1500 rows of 12000 take 28 us in one group, 36 in two).
constexpr int STREAM_WIDTH_MAX = 8 * 32 * 64;
int stream_groups(int width, bool bare) { return width <= 2 * 32 * 32 ? 8 : width <= 4 * 32 * 32 ? 4 : width <= 8 * 32 * 32 || bare ? 2 : 1; }
template <typename T>
StreamKernel stream_kernel(int width, bool bare)
{
    switch (stream_groups(width, bare)) {
    case 8: return rms_stream_kernel<T, 2, 32>;
    case 4: return rms_stream_kernel<T, 4, 32>;
    case 2: return width <= 8 * 32 * 32 ? rms_stream_kernel<T, 8, 32> : rms_stream_kernel<T, 8, 64>;
    default: return rms_stream_kernel<T, 16, 32>;
    }
}
bool bare(const RmsArgs &a) { return !a.r && !a.g; }

// Shared-memory opt-in of the current device, once.
int stream_opt_in()
{
    static std::atomic<int> done[MAX_DEVICES];
    const int dev = current_device_slot();
    if (dev < 0) { set_error("irms_quant: no current device, or its index is beyond %d", MAX_DEVICES - 1); return ICONV_ERR_UNSUPPORTED; }
    if (!done[dev].load(std::memory_order_acquire)) {
        for (int width = 2048; width <= STREAM_WIDTH_MAX; width *= 2)
            for (bool b : {false, true})
                for (StreamKernel k : {stream_kernel<float>(width, b), stream_kernel<__half>(width, b), stream_kernel<__nv_bfloat16>(width, b)})
                    ICONV_CUDA_TRY(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM));
        done[dev].store(1, std::memory_order_release);
    }
    return ICONV_OK;
}
// The current device's SM count; 0 where it cannot be had.
int sm_count()
{
    static std::atomic<int> count[MAX_DEVICES];
    const int dev = current_device_slot();
    if (dev < 0) return 0;
    int n = count[dev].load(std::memory_order_relaxed);
    if (n == 0 && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) count[dev].store(n, std::memory_order_relaxed);
    return n;
}

// Rows of 8 KB or more, with a residual 16 KB (there a block per row has enough in flight: 8192 rows of 4096 in bfloat16 take 38 us so, 44 as a
// stream; without the residual 27 and 27, 4096 rows of 8192 36 and 28), of which the ring takes one for every group and three at least; four
// rows or more for every SM.
bool streams(const RmsArgs &a, int element)
{
    const long long bytes = (long long)a.width * element, most = MAX_SMEM - (long long)sizeof(StreamShared);
    const bool residual = a.r != nullptr;
    if (bytes < (residual ? 16384 : 8192) || a.width > STREAM_WIDTH_MAX || std::max(3, stream_groups(a.width, bare(a))) * bytes * (residual ? 2 : 1) > most) return false;
    const int sms = sm_count();
    return sms > 0 && a.rows >= 4ll * sms;
}

template <typename T>
int launch_stream(const RmsArgs &a, cudaStream_t stream)
{
    const int rc = stream_opt_in(), sms = sm_count();
    if (rc != ICONV_OK) return rc;
    StreamArgs s;
    s.a = a;
    s.row_bytes = a.width * (int)sizeof(T);
    s.stage_bytes = s.row_bytes * (a.r ? 2 : 1);
    const int groups = stream_groups(a.width, bare(a));
    s.stages = std::min((MAX_SMEM - (int)sizeof(StreamShared)) / s.stage_bytes, STREAM_STAGES_MAX) / groups * groups;
    s.status = device_status_ptr();
    if (!s.status) { set_error("device status word not available"); return ICONV_ERR_CUDA; }
    const auto kernel = stream_kernel<T>(a.width, bare(a));
    ICONV_CUDA_TRY(launch_kernel(kernel, true, (unsigned)std::min<long long>(a.rows, sms), 32 * (STREAM_WARPS + STREAM_LOADERS),
                                 (size_t)s.stages * s.stage_bytes + sizeof(StreamShared), stream, s));
    return ICONV_OK;
}

template <typename T>
int launch_rms(const RmsArgs &a, bool whole, cudaStream_t stream)
{
    constexpr int VE = 16 / (int)sizeof(T);
    if (whole && streams(a, (int)sizeof(T))) return launch_stream<T>(a, stream);
    if constexpr (sizeof(T) == 2) {
        ShiftArgs s;
        if (!whole && shift_args<T>(a, s)) {
            ICONV_CUDA_TRY(launch_shift<T>(s, stream));
            return ICONV_OK;
        }
    }
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
    if (d.width > (1 << 24)) { set_error("irms_quant: width beyond 2^24"); return ICONV_ERR_SHAPE; }
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
