// Products of a handful of 8-bit rows (imat_forward with at most 16 tokens): the weights stream from memory into registers.
//
// What bounds such a call is the weights' way from HBM and, below some 20 MB of them, latency.  The tensor-memory kernels need a chain of
// set-up, descriptor fetches, one load instruction after another (350 cycles each) and barriers before the first byte is used; here
// every warp asks for its first 8 KB of weights straight away, before it waits for the kernel ahead in the stream, and the
// arithmetic -- two or four instructions per 512 bytes -- is nothing beside the loads.  The warp-level tensor instruction (m16n8k32)
// is wide enough for that.
//
// The layout is the plan's: blocks of 128 rows x 128 bytes.  A block of this kernel owns 32 consecutive packed rows (32 channels, or the gate and
// the up projection of 16) and its warps share the reduction.  The order of k inside an instruction is free as long as weights and rows agree:
// lane (g, t) takes the 16 bytes at 16 t of rows g, g + 8, g + 16, g + 24 of the weights and of token g of the rows, which serve two instructions.
// Whole numbers: the warps' sums meet in shared memory, in any order the same.
#pragma once

#include "mat_device.cuh"

namespace iconv {

constexpr int MAT_STREAM_ROWS = 32, MAT_STREAM_WARPS_MAX = 16, MAT_STREAM_TOKENS = 16;
constexpr int MAT_STREAM_AT_ONCE = 2;            // blocks of 128 bytes of the reduction that a warp has in flight: 8 KB of weights
constexpr int MAT_STREAM_PITCH = 36;             // words between two tokens of the sums in shared memory: the fragments' stores meet no bank twice

constexpr int MAT_STREAM_SMEM = MAT_STREAM_WARPS_MAX * MAT_STREAM_TOKENS * MAT_STREAM_PITCH * 4;

__device__ __forceinline__ uint4 ld_weights(const int8_t *p)      // (a plan's constants, used once: they need no place in L1)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void mma_s8(int (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct MatStreamArgs {
    const int8_t *packed;
    const int8_t *x;
    long long x_stride;
    int last_chunk;                 // (k - 1) / 16 * 16: where the last 16 bytes of a row start
};

// TOKENS8: groups of eight tokens.
template <typename T, bool GATED, int TOKENS8>
__global__ void __launch_bounds__(32 * MAT_STREAM_WARPS_MAX)
mat_stream_kernel(const __grid_constant__ MatStreamArgs s, const __grid_constant__ MatArgs a)
{
    extern __shared__ int sums[];                // [warps][tokens][MAT_STREAM_PITCH]
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), warps = (int)(blockDim.x >> 5);
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int row0 = (int)blockIdx.x * MAT_STREAM_ROWS;                          // first packed row
    const int kb0 = a.k_blocks * warp / warps, kb1 = a.k_blocks * (warp + 1) / warps;
    const int8_t *w = s.packed + ((long long)(row0 / BLOCK_M) * a.k_blocks * BLOCK_M + row0 % BLOCK_M + g) * 128 + t * 16;
    const int8_t *xr[TOKENS8];
#pragma unroll
    for (int q = 0; q < TOKENS8; ++q) xr[q] = s.x + (long long)(q * 8 + g < a.m ? q * 8 + g : a.m - 1) * s.x_stride;      // (columns beyond the last token are not stored)
    const float2 par = __ldg(a.row_params + row0 + lane);
    grid_dep_launch();

    int acc[2][TOKENS8][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int q = 0; q < TOKENS8; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][q][e] = 0;

    bool first = true;
    for (int kb = kb0; kb < kb1; kb += MAT_STREAM_AT_ONCE) {
        uint4 wv[MAT_STREAM_AT_ONCE][2][4], xv[MAT_STREAM_AT_ONCE][2][TOKENS8];
#pragma unroll
        for (int b = 0; b < MAT_STREAM_AT_ONCE; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) wv[b][h][i] = ld_weights(w + (long long)(kb + b < kb1 ? kb + b : kb) * MAT_BLOCK + i * 1024 + h * 64);
        if (first) grid_dep_wait();              // the rows may come from the kernel before this one
        first = false;
#pragma unroll
        for (int b = 0; b < MAT_STREAM_AT_ONCE; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k0 = (kb + b) * 128 + h * 64 + t * 16;                 // (beyond the end the weights are zeros: any bytes will do)
#pragma unroll
                for (int q = 0; q < TOKENS8; ++q) xv[b][h][q] = ld_tensor((const uint4 *)(xr[q] + (k0 < s.last_chunk ? k0 : s.last_chunk)));
            }
#pragma unroll
        for (int b = 0; b < MAT_STREAM_AT_ONCE; ++b) {
            if (kb + b >= kb1) break;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint4 lo = wv[b][h][2 * i], hi = wv[b][h][2 * i + 1];
#pragma unroll
                    for (int q = 0; q < TOKENS8; ++q) {
                        const uint4 xq = xv[b][h][q];
                        mma_s8(acc[i][q], lo.x, hi.x, lo.y, hi.y, xq.x, xq.y);
                        mma_s8(acc[i][q], lo.z, hi.z, lo.w, hi.w, xq.z, xq.w);
                    }
                }
        }
    }
    if (first) grid_dep_wait();

    int *mine = sums + warp * (TOKENS8 * 8) * MAT_STREAM_PITCH;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int q = 0; q < TOKENS8; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[(q * 8 + 2 * t + (e & 1)) * MAT_STREAM_PITCH + i * 16 + (e >> 1) * 8 + g] = acc[i][q][e];
    __syncthreads();
    // a warp per token, a lane per packed row
    const int ch = GATED ? (int)blockIdx.x * 16 + (lane & 15) : row0 + lane;
    const bool stores = ch < a.n && (!GATED || lane < 16);
    for (int tok = warp; tok < (int)a.m; tok += warps) {
        const float sx = __uint_as_float(ld_tensor((const unsigned *)a.x_scales + tok));
        float res = 0.0f;
        if (!GATED && a.residual && stores) res = mat_value<T>(((const T *)a.residual)[tok * a.ld_res + ch]);
        int total = 0;
        for (int i = 0; i < warps; ++i) total += sums[(i * (TOKENS8 * 8) + tok) * MAT_STREAM_PITCH + lane];
        float y[1] = {fmaf(__fmul_rn((float)total, par.x), sx, par.y)};
        if (GATED) {
            const float up = __shfl_xor_sync(0xffffffffu, y[0], 16);
            mat_act<sizeof(T) == 4, 1>(a.act, y);
            y[0] = __fmul_rn(y[0], up);
        } else {
            mat_act<sizeof(T) == 4, 1>(a.act, y);
            if (a.residual) y[0] = __fadd_rn(y[0], res);
        }
        if (stores) ((T *)a.out)[tok * a.ld_out + ch] = mat_round<T>(y[0]);
    }
}

}  // namespace iconv
