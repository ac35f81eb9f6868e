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
//   mat_few_kernel    few tokens: one tile of 128 channels x up to 128 tokens per cluster of 1, 2, 4 or 8 CTAs, which share the reduction
//                     and add their int32 parts through distributed shared memory (whole numbers: the order does not matter, nothing is kept
//                     in global memory, two calls share nothing).
//
// In both a warp loads the weights (before it waits for the kernel ahead in the stream: they are constants), another the rows, a third
// issues the instructions, eight run the epilogue.  All waits are bounded as in the convolution kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "umma_device.cuh"

namespace iconv {

constexpr int MAT_BLOCK = BLOCK_M * 128;          // bytes of a weight block
constexpr int MAT_EPI_WARPS = 8;
constexpr int MAT_THREADS = 32 * (EPI_WARP0 + MAT_EPI_WARPS);
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
    unsigned long long drain;
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

// y / (1 + exp(-z)): both smooth activations but one are of this form
__device__ __forceinline__ float mat_sigmoid_times(float y, float z) { return __fdividef(y, 1.0f + __expf(-z)); }

template <int N>
__device__ __forceinline__ void mat_act(int act, float (&y)[N])
{
    switch (act) {
    case IMAT_RELU:
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = y[j] < 0.0f ? 0.0f : y[j];      // (a NaN stays one)
        break;
    case IMAT_SILU:
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = mat_sigmoid_times(y[j], y[j]);
        break;
    case IMAT_GELU:
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = 0.5f * y[j] * (1.0f + erff(y[j] * 0.70710678118654752f));
        break;
    case IMAT_GELU_TANH:            // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u))
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = mat_sigmoid_times(y[j], y[j] * fmaf(0.0713548162726f, y[j] * y[j], 1.5957691216057f));
        break;
    default: break;
    }
}

// Scales of the 16 tokens from tok0 on (0 beyond the last): the same for every lane.
__device__ __forceinline__ void mat_scales16(const MatArgs &a, long long tok0, float (&sx)[16])
{
    if (tok0 + 16 <= a.m) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 w = ld_tensor((const uint4 *)(a.x_scales + tok0) + j);
            sx[4 * j] = __uint_as_float(w.x); sx[4 * j + 1] = __uint_as_float(w.y); sx[4 * j + 2] = __uint_as_float(w.z); sx[4 * j + 3] = __uint_as_float(w.w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) sx[j] = tok0 + j < a.m ? __uint_as_float(ld_tensor((const unsigned *)a.x_scales + tok0 + j)) : 0.0f;
    }
}

// This lane's channel of its channel tile (quad: the warp's quarter of the accumulator's lanes).
template <bool GATED>
__device__ __forceinline__ int mat_channel(int ch_tile, int quad, int lane)
{
    return GATED ? ch_tile * 64 + quad * 16 + (lane & 15) : ch_tile * 128 + quad * 32 + lane;
}

// 16 columns of an accumulator at t_addr: tokens tok0 ... of the lane's channel.
template <typename T, bool GATED>
__device__ __forceinline__ void mat_columns(const MatArgs &a, uint32_t t_addr, long long tok0, int ch, float2 par, int lane)
{
    const bool ch_ok = ch < a.n;
    const int count = a.m - tok0 < 16 ? (int)(a.m - tok0) : 16;
    float sx[16];
    mat_scales16(a, tok0, sx);
    T *out = (T *)a.out + tok0 * a.ld_out + ch;
    if (!GATED) {
        float res[16];
        const bool add = a.residual != nullptr;
        if (add) {
            const T *r = (const T *)a.residual + tok0 * a.ld_res + ch;
#pragma unroll
            for (int j = 0; j < 16; ++j) res[j] = ch_ok && j < count ? mat_value<T>(r[j * a.ld_res]) : 0.0f;
        }
        int acc[16];
        tmem_ld16_sync(t_addr, acc);
        float y[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = fmaf((float)acc[j] * par.x, sx[j], par.y);
        mat_act<16>(a.act, y);
        if (add)
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] += res[j];
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (ch_ok && j < count) out[j * a.ld_out] = mat_round<T>(y[j]);
    } else {
        int acc[16];
        tmem_ld16_sync(t_addr, acc);
        const bool up_lane = lane >= 16;            // lanes 0-15 hold the gate of 16 channels, lanes 16-31 their up projection
        float g[8], u[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            // two tokens: the lower lanes finish the first, the upper lanes the second
            const float v0 = fmaf((float)acc[2 * p] * par.x, sx[2 * p], par.y), v1 = fmaf((float)acc[2 * p + 1] * par.x, sx[2 * p + 1], par.y);
            const float other = __shfl_xor_sync(0xffffffffu, up_lane ? v0 : v1, 16);
            g[p] = up_lane ? other : v0;
            u[p] = up_lane ? v1 : other;
        }
        mat_act<8>(a.act, g);
        out += up_lane ? a.ld_out : 0;
#pragma unroll
        for (int p = 0; p < 8; ++p)
            if (ch_ok && 2 * p + (up_lane ? 1 : 0) < count) out[2 * p * a.ld_out] = mat_round<T>(g[p] * u[p]);
    }
}

// What both kernels set up; `consumers` epilogue warps give an accumulator back.
template <bool PAIR>
__device__ __forceinline__ uint32_t mat_set_up(MatShared *sh, const MatArgs &a, int warp, int consumers)
{
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(smem_u32(&sh->full[s]), 2);               // the loader of the weights and the loader of the rows
            mbar_init(smem_u32(&sh->empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sh->tmem_full[b]), 1);
            mbar_init(smem_u32(&sh->tmem_empty[b]), (uint32_t)consumers);
        }
        mbar_init(smem_u32(&sh->drain), 1);
        sh->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        grid_dep_launch();
    }
    if (warp == MMA_WARP) {
        if (PAIR) tmem_alloc_pair(smem_u32(&sh->tmem_base), (uint32_t)a.tmem_cols);
        else tmem_alloc(smem_u32(&sh->tmem_base), (uint32_t)a.tmem_cols);
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();                // the peer's barriers exist before anything arrives at them
    tc_fence_after();
    return sh->tmem_base;
}

// After an abort: wait (bounded) for what this warp's lane 0 may have in flight.
template <bool PAIR>
__device__ __forceinline__ void mat_drain(MatShared *sh, int warp, int lane, int last_stage, uint32_t last_parity, bool issues)
{
    volatile int never = 0;
    if (warp < 2 && lane == 0) {
        if (last_stage >= 0) mbar_wait(smem_u32(&sh->full[last_stage]), last_parity, &never);
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
__global__ void __launch_bounds__(MAT_THREADS, 1)
mat_bulk_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ MatArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    MatShared *sh = (MatShared *)(tiles + (size_t)a.stages * a.stage_bytes);
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const uint32_t rank = __shfl_sync(0xffffffffu, cluster_rank(), 0);
    const int ch_pairs = (a.ch_tiles + 1) >> 1;
    const long long num_tiles = (long long)ch_pairs * a.tok_tiles;
    const long long tile0 = blockIdx.x >> 1, tile_step = gridDim.x >> 1;
    const int half = a.nt >> 1;                  // tokens that each CTA of the pair brings
    if (threadIdx.x == 32) {
        prefetch_tensormap(&tmap_w);
        prefetch_tensormap(&tmap_x);
    }
    const uint32_t tmem_base = mat_set_up<true>(sh, a, warp, 2 * MAT_EPI_WARPS);

    // tile -> channel pair, token tile: token tiles in groups of MAT_GROUP, within a group all of them for one channel pair after another
    auto place = [&](long long tile, int &cp, int &tt) {
        const long long per_group = (long long)ch_pairs * MAT_GROUP;
        const int g = (int)(tile / per_group);
        const int in = (int)(tile - g * per_group);
        const int width = a.tok_tiles - g * MAT_GROUP < MAT_GROUP ? a.tok_tiles - g * MAT_GROUP : MAT_GROUP;
        cp = in / width;
        tt = g * MAT_GROUP + in - cp * width;
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
            bool ok = true;
            for (long long tile = tile0; tile < num_tiles && ok; tile += tile_step) {
                int cp, tt;
                place(tile, cp, tt);
                const int ct = 2 * cp + (int)rank < a.ch_tiles ? 2 * cp + (int)rank : a.ch_tiles - 1;   // (an odd last tile's partner loads it too; its results are not stored)
                int row = warp == 0 ? ct * a.k_blocks * BLOCK_M : 0;
                const int tok = tt * a.nt + (int)rank * half;
                for (int kb = 0; kb < a.k_blocks; ++kb, row += BLOCK_M) {
                    if (!mbar_wait(smem_u32(&sh->empty[stage]), parity ^ 1u, &sh->abort_flag)) {
                        mat_give_up(sh, a.status, 1);
                        ok = false;
                        break;
                    }
                    const uint32_t full = smem_u32(&sh->full[stage]);
                    const uint32_t dst = smem_u32(tiles + (size_t)stage * a.stage_bytes);
                    if (rank == 0) mbar_expect_tx(full, bytes);
                    if (warp == 0) tma_load_2d_pair(dst, &tmap_w, full & PEER_MASK, 0, row);
                    else tma_load_2d_pair(dst + MAT_BLOCK, &tmap_x, full & PEER_MASK, kb * 128, tok);
                    last_stage = stage;
                    last_parity = parity;
                    if (++stage == a.stages) { stage = 0; parity ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == MMA_WARP) {
        // ---------------------------------------------------------------- MMA issuer
        if (rank == 0) {
            const uint32_t a_lo0 = ((smem_u32(tiles) & 0x3FFFFu) >> 4) | (1u << 16);
            IssueRing ring;
            ring.stage = 0; ring.parity = 0; ring.a_lo = a_lo0;
            ring.full_bar = smem_u32(&sh->full[0]); ring.empty_bar = smem_u32(&sh->empty[0]);
            int t = 0;
            for (long long tile = tile0; tile < num_tiles; tile += tile_step, ++t) {
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
        for (long long tile = tile0; tile < num_tiles; tile += tile_step, ++t) {
            const int buf = t & 1;
            int cp, tt;
            place(tile, cp, tt);
            const int ct = 2 * cp + (int)rank;
            const int ch = mat_channel<GATED>(ct, quad, lane);
            const float2 par = ct < a.ch_tiles ? __ldg(a.row_params + (size_t)ct * BLOCK_M + quad * 32 + lane) : make_float2(0.0f, 0.0f);
            if (!mbar_wait_warp(smem_u32(&sh->tmem_full[buf]), (uint32_t)((t >> 1) & 1), &sh->abort_flag, lane)) {
                mat_give_up(sh, a.status, 4);
                break;
            }
            tc_fence_after();
            const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * MAT_BULK_TOKENS);
            for (int c = part; c < (a.nt >> 4); c += 2) {
                const long long tok0 = (long long)tt * a.nt + c * 16;
                if (tok0 >= a.m) break;
                mat_columns<T, GATED>(a, t_row + (uint32_t)(c * 16), tok0, ch, par, lane);
            }
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
__device__ __forceinline__ int mat_peer_load(uint32_t addr)
{
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// SPLIT: CTAs of the cluster that share a tile's reduction.
template <typename T, bool GATED, int SPLIT>
__global__ void __launch_bounds__(MAT_THREADS, 1)
mat_few_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ MatArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    MatShared *sh = (MatShared *)(tiles + (size_t)a.stages * a.stage_bytes);
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const int rank = SPLIT > 1 ? (int)__shfl_sync(0xffffffffu, cluster_rank(), 0) : 0;
    const int tile = (int)(blockIdx.x / SPLIT);
    const int ct = tile / a.tok_tiles, tt = tile - ct * a.tok_tiles;      // (neighbours share the weights)
    const long long tok_first = (long long)tt * a.nt;
    const int kb0 = (int)((long long)a.k_blocks * rank / SPLIT), kb1 = (int)((long long)a.k_blocks * (rank + 1) / SPLIT);
    if (threadIdx.x == 32) {
        prefetch_tensormap(&tmap_w);
        prefetch_tensormap(&tmap_x);
    }
    const uint32_t tmem_base = mat_set_up<false>(sh, a, warp, MAT_EPI_WARPS);

    int last_stage = -1;
    uint32_t last_parity = 0;
    const int quad = warp & 3, part = (warp - EPI_WARP0) >> 2;
    const int columns = a.m - tok_first < a.nt ? (int)(a.m - tok_first) : a.nt;        // tokens of this tile
    int *parts = (int *)tiles;                   // [tokens][128 lanes] of this CTA's part of the sums, where the stages were
    if (warp < 2) {
        if (lane == 0) {
            if (warp == 1) grid_dep_wait();                     // the rows may come from the kernel before this one
            const uint32_t bytes = (uint32_t)(warp == 0 ? MAT_BLOCK : a.nt * 128);
            int stage = 0;
            uint32_t parity = 0;
            int row = (ct * a.k_blocks + kb0) * BLOCK_M;
            for (int kb = kb0; kb < kb1; ++kb, row += BLOCK_M) {
                if (!mbar_wait(smem_u32(&sh->empty[stage]), parity ^ 1u, &sh->abort_flag)) {
                    mat_give_up(sh, a.status, 1);
                    break;
                }
                const uint32_t full = smem_u32(&sh->full[stage]);
                const uint32_t dst = smem_u32(tiles + (size_t)stage * a.stage_bytes);
                mbar_expect_tx(full, bytes);
                if (warp == 0) tma_load_2d(dst, &tmap_w, full, 0, row);
                else tma_load_2d(dst + MAT_BLOCK, &tmap_x, full, kb * 128, (int)tok_first);
                last_stage = stage;
                last_parity = parity;
                if (++stage == a.stages) { stage = 0; parity ^= 1u; }
            }
        }
        __syncwarp();
    } else if (warp == MMA_WARP) {
        const uint32_t a_lo0 = ((smem_u32(tiles) & 0x3FFFFu) >> 4) | (1u << 16);
        IssueRing ring;
        ring.stage = 0; ring.parity = 0; ring.a_lo = a_lo0;
        ring.full_bar = smem_u32(&sh->full[0]); ring.empty_bar = smem_u32(&sh->empty[0]);
        if (!issue_rounds<false>(ring, tmem_base, a.idesc, kb1 - kb0, a.stages, a_lo0, (uint32_t)a.stage_bytes >> 4, MAT_BLOCK >> 4, MAT_DESC_HI,
                                 smem_u32(&sh->full[0]), smem_u32(&sh->empty[0]), &sh->abort_flag))
            mat_give_up(sh, a.status, 3);
        else if (elect_one()) umma_commit(smem_u32(&sh->tmem_full[0]));
        __syncwarp();
    } else if (warp >= EPI_WARP0) {
        grid_dep_wait();
        const int ch = mat_channel<GATED>(ct, quad, lane);
        const float2 par = __ldg(a.row_params + (size_t)ct * BLOCK_M + quad * 32 + lane);
        const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16);
        if (!mbar_wait_warp(smem_u32(&sh->tmem_full[0]), 0, &sh->abort_flag, lane)) {
            mat_give_up(sh, a.status, 4);
        } else {
            tc_fence_after();
            for (int c = part; c * 16 < columns; c += 2) {
                if (SPLIT == 1) {
                    mat_columns<T, GATED>(a, t_row + (uint32_t)(c * 16), tok_first + c * 16, ch, par, lane);
                } else {
                    int acc[16];
                    tmem_ld16_sync(t_row + (uint32_t)(c * 16), acc);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c * 16 + j < columns) parts[(c * 16 + j) * BLOCK_M + quad * 32 + lane] = acc[j];
                }
            }
        }
        __syncwarp();
    } else {
        grid_dep_wait();                         // (no thread of the grid may be gone before the kernel ahead is done)
    }

    tc_fence_before();
    __syncthreads();
    if (sh->abort_flag) {
        mat_drain<false>(sh, warp, lane, last_stage, last_parity, true);
        __syncthreads();
    }
    if (SPLIT > 1) {
        cluster_sync_all();                      // every CTA's part is written
        if (warp >= EPI_WARP0) {
            // columns rank, rank + SPLIT, ... in turn by the two groups of four warps
            const int ch = mat_channel<GATED>(ct, quad, lane);
            const float2 par = __ldg(a.row_params + (size_t)ct * BLOCK_M + quad * 32 + lane);
            uint32_t from[SPLIT];
#pragma unroll
            for (int r = 0; r < SPLIT; ++r) from[r] = mat_peer_address(smem_u32(parts) + (uint32_t)((quad * 32 + lane) * 4), (uint32_t)r);
            for (int c = rank + part * SPLIT; c < columns; c += 2 * SPLIT) {
                const long long tok = tok_first + c;
                const bool mine = ch < a.n && (!GATED || lane < 16);
                const float sx = __uint_as_float(ld_tensor((const unsigned *)a.x_scales + tok));
                float res = 0.0f;
                if (!GATED && a.residual && mine) res = mat_value<T>(((const T *)a.residual)[tok * a.ld_res + ch]);
                int acc = 0;
#pragma unroll
                for (int r = 0; r < SPLIT; ++r) acc += mat_peer_load(from[r] + (uint32_t)(c * BLOCK_M * 4));
                float y[1] = {fmaf((float)acc * par.x, sx, par.y)};
                if (GATED) {
                    const float up = __shfl_xor_sync(0xffffffffu, y[0], 16);
                    mat_act<1>(a.act, y);
                    y[0] *= up;
                } else {
                    mat_act<1>(a.act, y);
                    y[0] += res;
                }
                if (mine) ((T *)a.out)[tok * a.ld_out + ch] = mat_round<T>(y[0]);
            }
        }
        cluster_sync_all();                      // no CTA leaves while another reads its part
    }
    if (warp == MMA_WARP) {
        tc_fence_after();
        tmem_dealloc(tmem_base, (uint32_t)a.tmem_cols);
    }
}

}  // namespace iconv
