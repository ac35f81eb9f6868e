// Products of 8-bit rows with int8 weights on the tensor cores (imat_forward): device code.
//
//   acc[c][t] = sum_k W[c][k] * X[t][k]      int32, exact
//   y = act(acc * sw[c] * sx[t] + b[c]) + residual[t][c]          or, gated, act(gate) * up
//
// The weights are the A operand (128 output channels are the 128 lanes of an accumulator), the rows (tokens) the B operand (the
// accumulator's columns).  So a few tokens make narrow instructions over whole weight tiles, which is what streaming the weights needs; an
// epilogue lane owns one channel, with its scale and bias in registers; and a warp's store of one token is 32 consecutive channels, with no
// staging.  The weights were laid out by the plan in blocks of 128 rows x 128 bytes (16 KB, one TMA load each); for a gated product the
// rows of a block alternate, 16 of the gate and 16 of the up projection, so that gate and up of a channel sit 16 lanes apart in one
// warp and meet in one shuffle: the main loop is that of a plain product.
//
// Two kernels.
//   mat_bulk_kernel   many tokens: persistent CTA pairs (cta_group::2), 256 channels x up to 256 tokens a tile, two accumulators
//                     of 256 columns so that the epilogue of one tile overlaps the instructions of the next.  Each CTA brings its own 128
//                     channels and its own half of the tokens: 32 KB for 4 instructions of 128 cycles, half of what single CTAs would need.
//   mat_few_kernel    few tiles: one tile of 128 channels x up to 128 tokens per cluster of up to 8 CTAs, which share the reduction and send
//                     each other their int32 parts through distributed shared memory (whole numbers: the order does not matter,
//                     nothing is kept in global memory, two calls share nothing).
//
// In both a warp loads the weights, another the rows, a third issues the instructions, eight or sixteen run the epilogue.  The first round of
// weights is asked for before the wait for the kernel ahead in the stream (they are constants); nobody starts a bounded wait before that one is
// over, however long the kernel ahead takes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "umma_device.cuh"

namespace iconv {

constexpr int MAT_BLOCK = BLOCK_M * 128;          // bytes of a weight block
constexpr int MAT_BULK_EPI = 16, MAT_FEW_EPI = 8;     // epilogue warps
constexpr int MAT_BULK_THREADS = 32 * (EPI_WARP0 + MAT_BULK_EPI), MAT_FEW_THREADS = 32 * (EPI_WARP0 + MAT_FEW_EPI);
constexpr int MAT_STAGES_MAX = 12;
constexpr int MAT_BULK_TOKENS = 256;              // columns of an accumulator buffer of the bulk kernel
constexpr int MAT_GROUP = 8;                      // token tiles that are walked together (the rows and the weights of a round both stay in L2)

struct MatArgs {
    long long m;                    // tokens
    int n;                          // output channels
    int ch_tiles, tok_tiles;        // tiles of 128 channels (64 when gated); tiles of nt tokens
    int nt;                         // tokens of a tile
    int k_blocks;                   // 128-byte blocks of the reduction
    int stages, stage_bytes;
    int split, recv_bytes;          // few-tile kernel: parts of a tile's reduction; memory for the sums that other parts send
    int tmem_cols;
    unsigned idesc;
    int act;
    const float2 *row_params;       // per packed weight row: scale, bias
    const float *x_scales;
    const void *residual;           // or NULL
    void *out;
    long long ld_res, ld_out;
    int *status;
};

struct MatShared {
    unsigned long long full[MAT_STAGES_MAX], empty[MAT_STAGES_MAX];
    unsigned long long tmem_full[2], tmem_empty[2];
    unsigned long long recv, drain;
    uint32_t tmem_base;
    volatile int abort_flag;
};

__device__ __forceinline__ void mat_give_up(MatShared *sh, int *status, int code)
{
    sh->abort_flag = 1;
    atomicCAS(status, 0, code);
}

template <typename T> __device__ __forceinline__ float mat_value(T v);
template <> __device__ __forceinline__ float mat_value<float>(float v) { return v; }
template <> __device__ __forceinline__ float mat_value<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float mat_value<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T mat_round(float v);
template <> __device__ __forceinline__ float mat_round<float>(float v) { return v; }
template <> __device__ __forceinline__ __half mat_round<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 mat_round<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// 2^x and 1 / x to two steps, x normal; results that are no normal numbers are zero
__device__ __forceinline__ float mat_exp2(float x)
{
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
    return d;
}
__device__ __forceinline__ float mat_reciprocal(float x)
{
    float d;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
    return d;
}

// y / (1 + exp(-z)) of SiLU and tanh-GELU, as y e / (1 + e) for z < 0, e = exp(-|z|): neither the exponential nor the quotient leaves float's range.  FINE
// (float results): z as it is, expf, a reciprocal with a Newton step.  16-bit results: z / log 2; values under |y| 2^-126 are zero.
template <bool FINE>
__device__ __forceinline__ float mat_sigmoid_times(float y, float z)
{
    const float e = FINE ? expf(-fabsf(z)) : mat_exp2(-fabsf(z));
    const float d = __fadd_rn(1.0f, e);
    float r = mat_reciprocal(d);
    if (FINE) r = fmaf(r, fmaf(-d, r, 1.0f), r);
    return __fmul_rn(z < 0.0f ? __fmul_rn(y, e) : y, r);
}

// y / 2 * (1 + erf(y / sqrt 2)) = y / 2 * erfc(-y / sqrt 2), where the factor is e = erfc(|y| / sqrt 2) = exp(-y^2 / 2) (c1 t + c2 t^2 + ...), t = 1 / (1 + c |y|), for
// y < 0 and 2 - e for the others: nothing cancels on the negative side, where the value falls to nothing.  The polynomials are fits for these kernels: least
// squares over |y| of 0 ... 15, weighted anew until the error is even (Lawson's iteration).  FINE (float results): of the relative error, 7e-9 in exact arithmetic and 4e-7 at
// most in float.  16-bit results: of the error in units of 3e-7 for e and 5e-6 relative, the larger; 4e-7 for e and 1.9e-6 relative in float.  (CUDA's erfc for float results
// took 4096 x 1024 x 4096 from 33 us to 55.)
template <bool FINE>
__device__ __forceinline__ float mat_gelu(float y)
{
    const float half = __fmul_rn(0.5f, y);
    const float t = mat_reciprocal(fmaf(FINE ? 0.246f : 0.26f, fabsf(y), 1.0f));
    float p, e;
    if (FINE) {
        p = fmaf(t, 0.0419157145f, -0.181555882f);
        p = fmaf(t, p, 0.236114511f); p = fmaf(t, p, -0.0902956311f); p = fmaf(t, p, 0.134590968f); p = fmaf(t, p, 0.123590758f);
        p = fmaf(t, p, 0.157703434f); p = fmaf(t, p, 0.185537543f); p = fmaf(t, p, 0.196109322f); p = fmaf(t, p, 0.196289268f);
        e = expf(__fmul_rn(-half, y));
    } else {
        p = fmaf(t, -0.145882931f, 0.45747601f);
        p = fmaf(t, p, -0.211728841f); p = fmaf(t, p, 0.331641501f); p = fmaf(t, p, 0.147230836f); p = fmaf(t, p, 0.214217862f);
        p = fmaf(t, p, 0.207045531f);
        const float z = __fmul_rn(0.849321800f, y);        // z^2 = y^2 / 2 / log 2
        e = mat_exp2(-__fmul_rn(z, z));
    }
    e = __fmul_rn(__fmul_rn(t, p), e);
    return __fmul_rn(half, y < 0.0f ? e : __fadd_rn(2.0f, -e));
}

template <bool FINE, int N>
__device__ __forceinline__ void mat_act(int act, float (&y)[N])
{
    switch (act) {
    case IMAT_RELU:
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = y[j] < 0.0f ? 0.0f : y[j];      // (a NaN stays one)
        break;
    case IMAT_SILU:
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = mat_sigmoid_times<FINE>(y[j], FINE ? y[j] : __fmul_rn(1.44269504f, y[j]));
        break;
    case IMAT_GELU:
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = mat_gelu<FINE>(y[j]);
        break;
    case IMAT_GELU_TANH:            // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u))
#pragma unroll
        for (int j = 0; j < N; ++j)
            y[j] = mat_sigmoid_times<FINE>(y[j], __fmul_rn(y[j], fmaf(FINE ? 0.0713548162726f : 0.102943240f, __fmul_rn(y[j], y[j]), FINE ? 1.5957691216057f : 2.302208198f)));
        break;
    default: break;
    }
}

// This lane's channel of its channel tile (quad: the warp's quarter of the accumulator's lanes).
template <bool GATED>
__device__ __forceinline__ int mat_channel(int ch_tile, int quad, int lane)
{
    return GATED ? ch_tile * 64 + quad * 16 + (lane & 15) : ch_tile * 128 + quad * 32 + lane;
}

// The epilogue of P columns (tokens tok ... tok + P - 1 of the lane's channel) in steps that a caller can spread: what it reads from memory, then the rest.
// All of it is short code in rolled loops: a block of the few-tile kernel runs it a handful of times, and code that runs once is bound
// by its own fetch (one unrolled group of 16 columns took 1500 cycles for the first time, 600 when it was there).  Loads go to
// clamped addresses instead of behind a branch each, which would make every one wait for the one before it.
template <int P>
__device__ __forceinline__ void mat_load_scales(const MatArgs &a, long long tok, float (&sx)[P])
{
    if (tok + P <= a.m) {
#pragma unroll
        for (int j = 0; j < P / 4; ++j) {
            const uint4 w = ld_tensor((const uint4 *)(a.x_scales + tok) + j);
            sx[4 * j] = __uint_as_float(w.x); sx[4 * j + 1] = __uint_as_float(w.y); sx[4 * j + 2] = __uint_as_float(w.z); sx[4 * j + 3] = __uint_as_float(w.w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < P; ++j) sx[j] = __uint_as_float(ld_tensor((const unsigned *)a.x_scales + (tok + j < a.m ? tok + j : a.m - 1)));
    }
}
template <typename T, int P>
__device__ __forceinline__ void mat_load_residual(const MatArgs &a, long long tok, int ch, T (&res)[P])
{
    const T *r = (const T *)a.residual + tok * a.ld_res + (ch < a.n ? ch : a.n - 1);
    const int last = (int)(a.m - 1 - tok < P - 1 ? a.m - 1 - tok : P - 1);
#pragma unroll
    for (int j = 0; j < P; ++j) {
        res[j] = *r;
        r += j < last ? a.ld_res : 0;
    }
}
// Every product and sum from here to the rounding is one operation of its own or an fmaf: the compiler may fuse others, and not the same ones in every kernel, but
// a row is the same whichever kernel a call runs.
// What the lane stores, from the sums: y[j] of token tok + j, or, gated, of token tok + 2 j + (lane >= 16) for j < P / 2.
template <typename T, bool GATED, int P>
__device__ __forceinline__ void mat_values(const MatArgs &a, const int (&acc)[P], const float (&sx)[P], const T (&res)[P], float2 par, int lane, float (&y)[P])
{
#pragma unroll
    for (int j = 0; j < P; ++j) y[j] = fmaf(__fmul_rn((float)acc[j], par.x), sx[j], par.y);
    if (!GATED) {
        mat_act<sizeof(T) == 4, P>(a.act, y);
        if (a.residual)
#pragma unroll
            for (int j = 0; j < P; ++j) y[j] = __fadd_rn(y[j], mat_value<T>(res[j]));
    } else {
        // lanes 0-15 hold the gate of 16 channels, lanes 16-31 their up projection: of two tokens the lower lanes finish the first, the upper ones the second
        const bool up_lane = lane >= 16;
        float g[P / 2], u[P / 2];
#pragma unroll
        for (int p = 0; p < P / 2; ++p) {
            const float other = __shfl_xor_sync(0xffffffffu, up_lane ? y[2 * p] : y[2 * p + 1], 16);
            g[p] = up_lane ? other : y[2 * p];
            u[p] = up_lane ? y[2 * p + 1] : other;
        }
        mat_act<sizeof(T) == 4, P / 2>(a.act, g);
#pragma unroll
        for (int p = 0; p < P / 2; ++p) y[p] = __fmul_rn(g[p], u[p]);
    }
}
// WHOLE: every token exists, and every lane's channel.
template <typename T, bool GATED, int P, bool WHOLE>
__device__ __forceinline__ void mat_store(const MatArgs &a, const float (&y)[P], long long tok, int ch, int lane)
{
    const int count = WHOLE ? P : ch < a.n ? (int)(a.m - tok < P ? a.m - tok : P) : 0;       // tokens that this lane stores
    const int first = GATED && lane >= 16 ? 1 : 0;
    T *out = (T *)a.out + (tok + first) * a.ld_out + ch;
    const long long step = GATED ? 2 * a.ld_out : a.ld_out;
#pragma unroll
    for (int j = 0; j < (GATED ? P / 2 : P); ++j) {
        if (WHOLE || (GATED ? 2 * j + first : j) < count) *out = mat_round<T>(y[j]);
        out += step;                        // (a product per store, behind its predicate, took twice as long)
    }
}

__device__ __forceinline__ void mat_tmem_ld8(uint32_t taddr, int (&r)[8])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
        : "r"(taddr)
        : "memory");
}

// A warp's share of a tile's epilogue: columns P part ... of every P `parts`.  What the next group reads is asked for before this one is
// stored, in the registers that it has just given free; the first group's is in hand (`begin`) while the accumulators are still being summed up.
template <typename T, bool GATED, int P>
struct MatColumns {
    float sx[P];
    T res[P];
    __device__ __forceinline__ void load(const MatArgs &a, long long tok, int ch)
    {
        mat_load_scales<P>(a, tok, sx);
        if (!GATED && a.residual) mat_load_residual<T, P>(a, tok, ch, res);
    }
    __device__ __forceinline__ void begin(const MatArgs &a, long long tok_first, int columns, int ch, int part)
    {
        if (part * P < columns) load(a, tok_first + part * P, ch);
    }
    __device__ __forceinline__ void run(const MatArgs &a, uint32_t t_row, long long tok_first, int columns, int ch, float2 par, int part, int parts, int lane)
    {
        const bool all = P == 16 && __all_sync(0xffffffffu, ch < a.n);
#pragma unroll 1
        for (int c = part * P; c < columns; c += parts * P) {
            int acc[P];
            float y[P];
            if constexpr (P == 8) mat_tmem_ld8(t_row + (uint32_t)c, acc);
            else tmem_ld16_sync(t_row + (uint32_t)c, acc);
            mat_values<T, GATED, P>(a, acc, sx, res, par, lane, y);
            if (c + parts * P < columns) load(a, tok_first + c + parts * P, ch);
            if (P == 16 && all && c + P <= columns) mat_store<T, GATED, P, true>(a, y, tok_first + c, ch, lane);
            else mat_store<T, GATED, P, false>(a, y, tok_first + c, ch, lane);
        }
    }
};

// Ask for a warp's residual rows of a tile (groups of P columns, every `parts`) while its sums are still being taken: from L2 they come in a third of
// the time.  A lane per token; its 32 channels are one line of 64 or 128 bytes, or two.
template <typename T, int P>
__device__ __forceinline__ void mat_prefetch_residual(const MatArgs &a, long long tok_first, int columns, int ch_first, int part, int parts, int lane)
{
    if (!a.residual || ch_first >= a.n) return;
    for (int c = part * P; c < columns; c += parts * P)
        if (lane < P && c + lane < columns)
            asm volatile("prefetch.global.L2 [%0];" ::"l"((const T *)a.residual + (tok_first + c + lane) * a.ld_res + ch_first));
}

// What both kernels set up; `consumers` epilogue warps give an accumulator back.  Warp 0 does the barriers, a lane each, and arms
// every stage for its first round (arms: this CTA's barriers count the loads; w_bytes, x_bytes: what a stage receives).
template <bool PAIR>
__device__ __forceinline__ uint32_t mat_set_up(MatShared *sh, const MatArgs &a, int warp, int lane, int consumers, bool arms, uint32_t w_bytes, uint32_t x_bytes, int blocks,
                                               uint32_t recv_bytes)
{
    if (warp == 0) {
        if (lane < a.stages) {
            mbar_init(smem_u32(&sh->full[lane]), 2);            // the loader of the weights and the loader of the rows
            mbar_init(smem_u32(&sh->empty[lane]), 1);
            if (arms && lane < blocks) {
                mbar_expect_tx(smem_u32(&sh->full[lane]), w_bytes);
                mbar_expect_tx(smem_u32(&sh->full[lane]), x_bytes);
            }
        } else if (lane >= 16 && lane < 18) {
            mbar_init(smem_u32(&sh->tmem_full[lane - 16]), 1);
            mbar_init(smem_u32(&sh->tmem_empty[lane - 16]), (uint32_t)consumers);
        } else if (lane == 18) {
            mbar_init(smem_u32(&sh->drain), 1);
            mbar_init(smem_u32(&sh->recv), 1);
            mbar_expect_tx(smem_u32(&sh->recv), recv_bytes);
            sh->abort_flag = 0;
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        if (PAIR) tmem_alloc_pair(smem_u32(&sh->tmem_base), (uint32_t)a.tmem_cols);
        else tmem_alloc(smem_u32(&sh->tmem_base), (uint32_t)a.tmem_cols);
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0) grid_dep_launch();     // (behind the tensor memory: see grid_dep_launch)
    if (PAIR) cluster_sync_all();                // the peer's barriers exist before anything arrives at them
    tc_fence_after();
    return sh->tmem_base;
}

// The loads of one block of the reduction into its stage: the weights' and the rows'.
template <bool PAIR>
__device__ __forceinline__ void mat_load_weights(const CUtensorMap *map, uint32_t dst, uint32_t full, int row)
{
    if (PAIR) tma_load_2d_pair(dst, map, full & PEER_MASK, 0, row);
    else tma_load_2d(dst, map, full, 0, row);
}
template <bool PAIR>
__device__ __forceinline__ void mat_load_rows(const CUtensorMap *map, uint32_t dst, uint32_t full, int kb, int tok)
{
    if (PAIR) tma_load_2d_pair(dst + MAT_BLOCK, map, full & PEER_MASK, kb * 128, tok);
    else tma_load_2d(dst + MAT_BLOCK, map, full, kb * 128, tok);
}

// After an abort: wait (bounded) for what this warp's lane 0 may have in flight.
template <bool PAIR>
__device__ __forceinline__ void mat_drain(MatShared *sh, int warp, int lane, int last_stage, uint32_t last_parity, bool issues)
{
    volatile int never = 0;
    if (warp != MMA_WARP && lane == 0 && last_stage >= 0) {
        mbar_wait(smem_u32(&sh->full[last_stage]), last_parity, &never);
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000) {}
    }
    if (warp == MMA_WARP && lane == 0 && issues) {
        if (PAIR) umma_commit_pair(smem_u32(&sh->drain)); else umma_commit(smem_u32(&sh->drain));
        mbar_wait(smem_u32(&sh->drain), 0, &never);
    }
}

constexpr uint32_t MAT_DESC_HI = (uint32_t)(((unsigned long long)(1024 >> 4) << 32 | (1ull << 46) | (2ull << 61)) >> 32);   // rows of 128 bytes, 128-byte swizzle, 8-row groups 1024 bytes apart

template <typename T, bool GATED>
__global__ void __launch_bounds__(MAT_BULK_THREADS, 1)
mat_bulk_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ MatArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    MatShared *sh = (MatShared *)(tiles + (size_t)a.stages * a.stage_bytes);
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const uint32_t rank = __shfl_sync(0xffffffffu, cluster_rank(), 0);
    const int ch_pairs = (a.ch_tiles + 1) >> 1;
    const unsigned num_tiles = (unsigned)ch_pairs * (unsigned)a.tok_tiles;       // (out has at most 2^40 elements)
    const unsigned tile0 = blockIdx.x >> 1, tile_step = gridDim.x >> 1;
    const int half = a.nt >> 1;                  // tokens that each CTA of the pair brings
    if (threadIdx.x == 32) {
        prefetch_tensormap(&tmap_w);
        prefetch_tensormap(&tmap_x);
    }
    const uint32_t tmem_base = mat_set_up<true>(sh, a, warp, lane, 2 * MAT_BULK_EPI, rank == 0, 2u * MAT_BLOCK, 2u * (uint32_t)half * 128u, a.stages, 0u);

    // tile -> channel pair, token tile: token tiles in groups of MAT_GROUP, within a group all of them for one channel pair after another
    auto place = [&](unsigned tile, int &cp, int &tt) {
        const unsigned per_group = (unsigned)ch_pairs * MAT_GROUP, g = tile / per_group, in = tile - g * per_group;
        const unsigned left = (unsigned)a.tok_tiles - g * MAT_GROUP, width = left < MAT_GROUP ? left : MAT_GROUP;
        cp = (int)(in / width);
        tt = (int)(g * MAT_GROUP + in) - cp * (int)width;
    };

    int last_stage = -1;
    uint32_t last_parity = 0;
    if (warp < 2) {
        // ---------------------------------------------------------------- loaders: warp 0 the weights, warp 1 the rows
        if (lane == 0) {
            if (warp == 1) grid_dep_wait();                     // the rows may come from the kernel before this one
            const uint32_t bytes = 2u * (uint32_t)(warp == 0 ? MAT_BLOCK : half * 128);     // both CTAs', counted on the leader's barrier
            int stage = 0;
            uint32_t parity = 0;
            bool ok = true, armed = true;                       // (the first round's barriers are)
            for (unsigned tile = tile0; tile < num_tiles && ok; tile += tile_step) {
                int cp, tt;
                place(tile, cp, tt);
                const int ct = 2 * cp + (int)rank < a.ch_tiles ? 2 * cp + (int)rank : a.ch_tiles - 1;   // (an odd last tile's partner loads it too; its results are not stored)
                int row = warp == 0 ? ct * a.k_blocks * BLOCK_M : 0;
                const int tok = tt * a.nt + (int)rank * half;
                for (int kb = 0; kb < a.k_blocks; ++kb, row += BLOCK_M) {
                    const uint32_t full = smem_u32(&sh->full[stage]);
                    const uint32_t dst = smem_u32(tiles + (size_t)stage * a.stage_bytes);
                    if (!armed) {
                        grid_dep_wait();
                        if (!mbar_wait(smem_u32(&sh->empty[stage]), parity ^ 1u, &sh->abort_flag)) {
                            mat_give_up(sh, a.status, 1);
                            ok = false;
                            break;
                        }
                        if (rank == 0) mbar_expect_tx(full, bytes);
                    }
                    if (warp == 0) mat_load_weights<true>(&tmap_w, dst, full, row);
                    else mat_load_rows<true>(&tmap_x, dst, full, kb, tok);
                    last_stage = stage;
                    last_parity = parity;
                    if (++stage == a.stages) { stage = 0; parity ^= 1u; armed = false; }
                }
            }
        }
        __syncwarp();
    } else if (warp == MMA_WARP) {
        // ---------------------------------------------------------------- MMA issuer
        grid_dep_wait();
        if (rank == 0) {
            const uint32_t a_lo0 = ((smem_u32(tiles) & 0x3FFFFu) >> 4) | (1u << 16);
            IssueRing ring;
            ring.stage = 0; ring.parity = 0; ring.a_lo = a_lo0;
            ring.full_bar = smem_u32(&sh->full[0]); ring.empty_bar = smem_u32(&sh->empty[0]);
            int t = 0;
            for (unsigned tile = tile0; tile < num_tiles; tile += tile_step, ++t) {
                const int buf = t & 1;
                if (!mbar_wait_warp(smem_u32(&sh->tmem_empty[buf]), (uint32_t)(((t >> 1) & 1) ^ 1), &sh->abort_flag, lane)) {
                    mat_give_up(sh, a.status, 2);
                    break;
                }
                tc_fence_after();
                if (!issue_rounds<true>(ring, tmem_base + (uint32_t)(buf * MAT_BULK_TOKENS), a.idesc, a.k_blocks, a.stages, a_lo0, (uint32_t)a.stage_bytes >> 4,
                                        MAT_BLOCK >> 4, MAT_DESC_HI, smem_u32(&sh->full[0]), smem_u32(&sh->empty[0]), &sh->abort_flag)) {
                    mat_give_up(sh, a.status, 3);
                    break;
                }
                if (elect_one()) umma_commit_pair(smem_u32(&sh->tmem_full[buf]));
            }
        }
        __syncwarp();
    } else if (warp >= EPI_WARP0) {
        // ---------------------------------------------------------------- epilogue
        grid_dep_wait();
        const int quad = warp & 3, part = (warp - EPI_WARP0) >> 2;
        int t = 0;
        for (unsigned tile = tile0; tile < num_tiles; tile += tile_step, ++t) {
            const int buf = t & 1;
            int cp, tt;
            place(tile, cp, tt);
            const int ct = 2 * cp + (int)rank;
            const int ch = mat_channel<GATED>(ct, quad, lane);
            const float2 par = ct < a.ch_tiles ? __ldg(a.row_params + (size_t)ct * BLOCK_M + quad * 32 + lane) : make_float2(0.0f, 0.0f);
            const long long tok_first = (long long)tt * a.nt;
            const int columns = a.m - tok_first < a.nt ? (int)(a.m - tok_first) : a.nt;
            if (!GATED) mat_prefetch_residual<T, 16>(a, tok_first, columns, ct * BLOCK_M + quad * 32, part, MAT_BULK_EPI / 4, lane);
            MatColumns<T, GATED, 16> share;
            share.begin(a, tok_first, columns, ch, part);
            if (!mbar_wait_warp(smem_u32(&sh->tmem_full[buf]), (uint32_t)((t >> 1) & 1), &sh->abort_flag, lane)) {
                mat_give_up(sh, a.status, 4);
                break;
            }
            tc_fence_after();
            const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * MAT_BULK_TOKENS);
            share.run(a, t_row, tok_first, columns, ch, par, part, MAT_BULK_EPI / 4, lane);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_leader(smem_u32(&sh->tmem_empty[buf]));
        }
        __syncwarp();
    }

    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (sh->abort_flag) {
        mat_drain<true>(sh, warp, lane, last_stage, last_parity, rank == 0);
        __syncthreads();
    }
    // neither CTA may leave (or give back its TMEM) while the other can still reach its shared memory or have instructions in flight that write its TMEM
    cluster_sync_all();
    if (warp == MMA_WARP) {
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, (uint32_t)a.tmem_cols);
    }
}

__device__ __forceinline__ uint32_t mat_peer_address(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// Four words into another CTA's shared memory, counted on that CTA's barrier.
__device__ __forceinline__ void mat_push(uint32_t addr, uint32_t bar, int x, int y, int z, int w)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
                 : "memory");
}
// Four columns each from two places, ready when it returns (load and wait in one statement: no register is looked at before).
__device__ __forceinline__ void mat_tmem_ld4x2(uint32_t t0, uint32_t t1, int (&r0)[4], int (&r1)[4])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%8];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%4, %5, %6, %7}, [%9];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r0[0]), "=r"(r0[1]), "=r"(r0[2]), "=r"(r0[3]), "=r"(r1[0]), "=r"(r1[1]), "=r"(r1[2]), "=r"(r1[3])
        : "r"(t0), "r"(t1)
        : "memory");
}

// Sums that a cluster shares: pieces of MAT_PIECE tokens are owned by its `split` parts in turn; a part sends the others' pieces to their
// owners as soon as its instructions are done (16 bytes a lane, received in memory of their own) and finishes its own.
constexpr int MAT_PIECE = 4;
constexpr int MAT_PIECE_BYTES = MAT_PIECE * 4 * BLOCK_M;

struct MatPart {                    // of a shared reduction: CTA `mine` of the cluster
    int mine, split, lg_split;
    int pieces, owned;
};
__device__ __forceinline__ MatPart mat_part(const MatArgs &a, int mine, int columns)
{
    MatPart p;
    p.mine = mine; p.split = a.split; p.lg_split = 31 - __clz(a.split);
    p.pieces = (columns + MAT_PIECE - 1) / MAT_PIECE;
    p.owned = p.pieces > mine ? (p.pieces - mine + p.split - 1) >> p.lg_split : 0;
    return p;
}

// What two of a part's pieces, numbers j and j + 1, read besides the sums.
template <typename T, bool GATED>
struct MatPieces {
    float sx0[4], sx1[4];
    T res0[4], res1[4];
    __device__ __forceinline__ void load(const MatArgs &a, const MatPart &p, long long tok_first, int j, int ch)
    {
        const int i0 = p.mine + (j << p.lg_split), i1 = j + 1 < p.owned ? i0 + p.split : i0;
        mat_load_scales<4>(a, tok_first + i0 * MAT_PIECE, sx0);
        mat_load_scales<4>(a, tok_first + i1 * MAT_PIECE, sx1);
        if (!GATED && a.residual) {
            mat_load_residual<T, 4>(a, tok_first + i0 * MAT_PIECE, ch, res0);
            mat_load_residual<T, 4>(a, tok_first + i1 * MAT_PIECE, ch, res1);
        }
    }
};

template <typename T, bool GATED>
__device__ __forceinline__ void mat_reduce(const MatArgs &a, MatShared *sh, const MatPart &p, MatPieces<T, GATED> &in, uint32_t recv, uint32_t t_row, long long tok_first,
                                           int ch, float2 par, int quad, int part, int lane)
{
    const uint32_t lane_off = (uint32_t)((quad * 32 + lane) * 16);
    const uint32_t bar = smem_u32(&sh->recv);
    // ---- send
#pragma unroll 1
    for (int c = part; c * 4 < p.pieces; c += 2) {
        int acc[16];
        tmem_ld16_sync(t_row + (uint32_t)(c * 16), acc);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = 4 * c + j, owner = i & (p.split - 1);
            if (i >= p.pieces || owner == p.mine) continue;
            // the owner's slots: [its pieces][the other parts]
            const int from = p.mine < owner ? p.mine : p.mine - 1;
            mat_push(mat_peer_address(recv + (uint32_t)(((i >> p.lg_split) * (p.split - 1) + from) * MAT_PIECE_BYTES) + lane_off, (uint32_t)owner),
                     mat_peer_address(bar, (uint32_t)owner),
                     acc[4 * j], acc[4 * j + 1], acc[4 * j + 2], acc[4 * j + 3]);
        }
    }
    // ---- finish this part's pieces, two at a time: numbers 2 part, 2 part + 1 of every four (what they read besides is in hand, or on its way)
    bool waited = false;
#pragma unroll 1
    for (int j = 2 * part; j < p.owned; j += 4) {
        const bool two = j + 1 < p.owned;
        const int i0 = p.mine + (j << p.lg_split), i1 = two ? i0 + p.split : i0;
        const long long tok0 = tok_first + i0 * MAT_PIECE, tok1 = tok_first + i1 * MAT_PIECE;
        int acc0[4], acc1[4];
        mat_tmem_ld4x2(t_row + (uint32_t)(i0 * MAT_PIECE), t_row + (uint32_t)(i1 * MAT_PIECE), acc0, acc1);
        if (!waited && !mbar_wait_warp(bar, 0, &sh->abort_flag, lane)) {
            mat_give_up(sh, a.status, 5);
            break;
        }
        waited = true;
        const uint32_t slot = recv + (uint32_t)(j * (p.split - 1) * MAT_PIECE_BYTES) + lane_off;
        const uint32_t second = two ? (uint32_t)((p.split - 1) * MAT_PIECE_BYTES) : 0u;
#pragma unroll 1
        for (int r = 0; r < p.split - 1; ++r) {
            const uint4 o = lds128(slot + (uint32_t)(r * MAT_PIECE_BYTES)), q = lds128(slot + second + (uint32_t)(r * MAT_PIECE_BYTES));
            acc0[0] += (int)o.x; acc0[1] += (int)o.y; acc0[2] += (int)o.z; acc0[3] += (int)o.w;
            acc1[0] += (int)q.x; acc1[1] += (int)q.y; acc1[2] += (int)q.z; acc1[3] += (int)q.w;
        }
        float y0[4], y1[4];
        mat_values<T, GATED, 4>(a, acc0, in.sx0, in.res0, par, lane, y0);
        mat_values<T, GATED, 4>(a, acc1, in.sx1, in.res1, par, lane, y1);
        if (j + 4 < p.owned) in.load(a, p, tok_first, j + 4, ch);
        mat_store<T, GATED, 4, false>(a, y0, tok0, ch, lane);
        if (two) mat_store<T, GATED, 4, false>(a, y1, tok1, ch, lane);
    }
}

// One tile per cluster of `split` CTAs that share its reduction.
template <typename T, bool GATED>
__global__ void __launch_bounds__(MAT_FEW_THREADS, 2)
mat_few_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ MatArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t recv = smem_u32(tiles) + (uint32_t)(a.stages * a.stage_bytes);
    MatShared *sh = (MatShared *)(tiles + (size_t)a.stages * a.stage_bytes + a.recv_bytes);
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const bool alone = a.split == 1;
    const int mine = alone ? 0 : (int)__shfl_sync(0xffffffffu, cluster_rank(), 0);       // this CTA's part of the reduction
    const int tile = (int)(blockIdx.x / (unsigned)a.split);
    const int ct = tile / a.tok_tiles, tt = tile - ct * a.tok_tiles;      // (neighbours share the weights)
    const long long tok_first = (long long)tt * a.nt;
    const int kb0 = (int)((long long)a.k_blocks * mine / a.split), kb1 = (int)((long long)a.k_blocks * (mine + 1) / a.split);
    const int columns = a.m - tok_first < a.nt ? (int)(a.m - tok_first) : a.nt;        // tokens of this tile
    if (threadIdx.x == 32) {
        prefetch_tensormap(&tmap_w);
        prefetch_tensormap(&tmap_x);
    }
    const MatPart shared = mat_part(a, mine, columns);
    const uint32_t tmem_base = mat_set_up<false>(sh, a, warp, lane, MAT_FEW_EPI, true, (uint32_t)MAT_BLOCK, (uint32_t)(a.nt * 128), kb1 - kb0,
                                                 (uint32_t)(shared.owned * (a.split - 1) * MAT_PIECE_BYTES));
    if (!alone) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");       // (waited for before the first word is sent)

    int last_stage = -1;
    uint32_t last_parity = 0;
    const int quad = warp & 3, part = (warp - EPI_WARP0) >> 2;
    const int w_row = (ct * a.k_blocks + kb0) * BLOCK_M;
    if (warp < 2) {
        // ---------------------------------------------------------------- loaders: warp 0 the weights, warp 1 the rows (from the second round on)
        if (lane == 0) {
            grid_dep_wait();                     // the rows may come from the kernel before this one
            const uint32_t bytes = (uint32_t)(warp == 0 ? MAT_BLOCK : a.nt * 128);
            int stage = 0;
            uint32_t parity = 1;
            for (int kb = kb0 + a.stages; kb < kb1; ++kb) {
                if (!mbar_wait(smem_u32(&sh->empty[stage]), parity ^ 1u, &sh->abort_flag)) {
                    mat_give_up(sh, a.status, 1);
                    break;
                }
                const uint32_t full = smem_u32(&sh->full[stage]), dst = smem_u32(tiles + (size_t)stage * a.stage_bytes);
                mbar_expect_tx(full, bytes);
                if (warp == 0) mat_load_weights<false>(&tmap_w, dst, full, w_row + (kb - kb0) * BLOCK_M);
                else mat_load_rows<false>(&tmap_x, dst, full, kb, (int)tok_first);
                last_stage = stage;
                last_parity = parity;
                if (++stage == a.stages) { stage = 0; parity ^= 1u; }
            }
        }
        __syncwarp();
        if (!alone) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    } else if (warp == MMA_WARP) {
        // ---------------------------------------------------------------- MMA issuer
        grid_dep_wait();
        const uint32_t a_lo0 = ((smem_u32(tiles) & 0x3FFFFu) >> 4) | (1u << 16);
        IssueRing ring;
        ring.stage = 0; ring.parity = 0; ring.a_lo = a_lo0;
        ring.full_bar = smem_u32(&sh->full[0]); ring.empty_bar = smem_u32(&sh->empty[0]);
        if (!issue_rounds<false>(ring, tmem_base, a.idesc, kb1 - kb0, a.stages, a_lo0, (uint32_t)a.stage_bytes >> 4, MAT_BLOCK >> 4, MAT_DESC_HI,
                                 smem_u32(&sh->full[0]), smem_u32(&sh->empty[0]), &sh->abort_flag))
            mat_give_up(sh, a.status, 3);
        else if (elect_one()) umma_commit(smem_u32(&sh->tmem_full[0]));
        __syncwarp();
        if (!alone) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    } else if (warp >= EPI_WARP0) {
        // ---------------------------------------------------------------- epilogue; before it the first round of loads, a warp's share each:
        // a lone thread needs 350 cycles per load instruction, and the weights need not wait for the kernel ahead
        const int first = kb1 - kb0 < a.stages ? kb1 - kb0 : a.stages;
        if (lane == 0)
            for (int i = warp - EPI_WARP0; i < first; i += MAT_FEW_EPI)
                mat_load_weights<false>(&tmap_w, smem_u32(tiles + (size_t)i * a.stage_bytes), smem_u32(&sh->full[i]), w_row + i * BLOCK_M);
        grid_dep_wait();
        if (lane == 0)
            for (int i = warp - EPI_WARP0; i < first; i += MAT_FEW_EPI) {
                mat_load_rows<false>(&tmap_x, smem_u32(tiles + (size_t)i * a.stage_bytes), smem_u32(&sh->full[i]), kb0 + i, (int)tok_first);
                last_stage = i;
            }
        __syncwarp();
        const int ch = mat_channel<GATED>(ct, quad, lane);
        const float2 par = __ldg(a.row_params + (size_t)ct * BLOCK_M + quad * 32 + lane);
        const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16);
        MatColumns<T, GATED, 8> share;
        MatPieces<T, GATED> pieces;
        if (!GATED && a.split == 1) mat_prefetch_residual<T, 8>(a, tok_first, columns, ct * BLOCK_M + quad * 32, part, MAT_FEW_EPI / 4, lane);
        if (a.split == 1) share.begin(a, tok_first, columns, ch, part);
        else if (2 * part < shared.owned) pieces.load(a, shared, tok_first, 2 * part, ch);
        const bool ok = mbar_wait_warp(smem_u32(&sh->tmem_full[0]), 0, &sh->abort_flag, lane);
        if (!alone) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        if (!ok) {
            mat_give_up(sh, a.status, 4);
        } else {
            tc_fence_after();
            if (a.split == 1) share.run(a, t_row, tok_first, columns, ch, par, part, MAT_FEW_EPI / 4, lane);
            else mat_reduce<T, GATED>(a, sh, shared, pieces, recv, t_row, tok_first, ch, par, quad, part, lane);
        }
        __syncwarp();
    } else {
        grid_dep_wait();
        if (!alone) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }

    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (sh->abort_flag) {
        mat_drain<false>(sh, warp, lane, last_stage, last_parity, true);
        __syncthreads();
    }
    // A CTA may leave once it has received all that is sent to it, which it has by now.  One that gave up waits for the others to end.
    if (!alone && sh->abort_flag) cluster_sync_all();
    if (warp == MMA_WARP) {
        tc_fence_after();
        tmem_dealloc(tmem_base, (uint32_t)a.tmem_cols);
    }
}

}  // namespace iconv
