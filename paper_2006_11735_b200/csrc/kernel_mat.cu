// Host side of the products of 8-bit rows with int8 weights (mat_device.cuh): validation, the plan's weight layout, which kernel and tile a
// call runs, the launch.
#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cstdio>
#include <cstring>
#include <new>

#include "mat_inst.h"

struct imat_plan_s {
    int n = 0, k = 0, out_dtype = 0, act = 0, gated = 0, device = -1, sms = 0;
    int ch_tiles = 0, k_blocks = 0;
    int8_t *packed = nullptr;              // [ch_tiles][k_blocks][128 rows][128 bytes]
    float2 *row_params = nullptr;          // [ch_tiles * 128] scale, bias
    CUtensorMap tmap_w;
};

namespace iconv {

namespace {

constexpr int MAT_K_MAX = 131071;          // 128 * 128 * k stays under 2^31

// What one call runs.
struct MatChoice {
    int split;                             // 0: bulk kernel
    int nt, tok_tiles, stages, stage_bytes, tmem_cols;
    unsigned grid;
    size_t smem;
};

struct PackArgs {
    const int8_t *w[2];
    const float *scales[2], *bias[2];
    long long w_stride;
    int n, k, gated, k_blocks, whole;      // whole: rows can be read 16 bytes at a time
    long long units;                       // 16-byte pieces of the layout
    int rows;                              // packed rows
    uint4 *packed;
    float2 *row_params;
};

// Packed row -> projection and channel.  Gated: rows alternate, 16 of the gate and 16 of the up projection.
__device__ __forceinline__ void pack_source(const PackArgs &a, int row, int &which, int &ch)
{
    which = a.gated ? (row >> 4) & 1 : 0;
    ch = a.gated ? (row >> 5) * 16 + (row & 15) : row;
}

// The plan's layout: every 16-byte piece (8 of a row of a block) from its row, zeros beyond the last channel and the end of the reduction.
__global__ void __launch_bounds__(256) mat_pack_kernel(const __grid_constant__ PackArgs a)
{
    const long long step = (long long)gridDim.x * blockDim.x;
    const long long first = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    for (long long u = first; u < a.units; u += step) {
        const long long block = u >> 10;                         // 128 rows of 8 pieces
        const int in = (int)(u & 1023);
        const long long ct = block / a.k_blocks;
        const int k0 = (int)(block - ct * a.k_blocks) * 128 + (in & 7) * 16;
        int which, ch;
        pack_source(a, (int)ct * BLOCK_M + (in >> 3), which, ch);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (ch < a.n && k0 < a.k) {
            const int8_t *src = a.w[which] + (long long)ch * a.w_stride + k0;
            if (a.whole && k0 + 16 <= a.k) {
                v = *(const uint4 *)src;
            } else {
                uint8_t b[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) b[j] = k0 + j < a.k ? (uint8_t)src[j] : 0;
                memcpy(&v, b, 16);
            }
        }
        a.packed[u] = v;
    }
    for (long long r = first; r < a.rows; r += step) {
        int which, ch;
        pack_source(a, (int)r, which, ch);
        a.row_params[r] = ch < a.n ? make_float2(a.scales[which][ch], a.bias[which] ? a.bias[which][ch] : 0.0f) : make_float2(0.0f, 0.0f);
    }
}

int round_up(int v, int to) { return (v + to - 1) / to * to; }

void stages_of(MatChoice &c, int room, int k_blocks)
{
    c.stages = std::min(std::min(room / c.stage_bytes, MAT_STAGES_MAX), std::max(k_blocks, 2));
    c.smem = 1024 + (size_t)c.stages * c.stage_bytes + sizeof(MatShared);
}

constexpr int MAT_ROOM = MAX_SMEM - 1024 - (int)sizeof(MatShared);

MatChoice choose_few(const imat_plan_t *p, long long rows)
{
    MatChoice c;
    c.tok_tiles = (int)((rows + 127) / 128);
    c.nt = round_up((int)((rows + c.tok_tiles - 1) / c.tok_tiles), 16);
    c.stage_bytes = MAT_BLOCK + c.nt * 128;
    c.tmem_cols = 32;
    while (c.tmem_cols < c.nt) c.tmem_cols *= 2;
    const long long tiles = (long long)p->ch_tiles * c.tok_tiles;
    c.split = 1;
    while (c.split < 8 && tiles * c.split * 2 <= p->sms + p->sms / 8 && p->k_blocks >= 4 * c.split) c.split *= 2;
    c.grid = (unsigned)(tiles * c.split);
    stages_of(c, MAT_ROOM, (p->k_blocks + c.split - 1) / c.split);
    const size_t parts = 1024 + (size_t)c.nt * BLOCK_M * 4 + sizeof(MatShared);      // a split tile's sums lie where the stages were
    while (c.split > 1 && c.smem < parts) { ++c.stages; c.smem += c.stage_bytes; }
    return c;
}

MatChoice choose_bulk(const imat_plan_t *p, long long rows)
{
    MatChoice c;
    c.split = 0;
    const long long pairs = p->sms / 2, ch_pairs = (p->ch_tiles + 1) / 2;
    long long best = -1;
    for (int nt = 256; nt >= 64; nt -= 32) {
        const long long tok_tiles = (rows + nt - 1) / nt, rounds = (ch_pairs * tok_tiles + pairs - 1) / pairs;
        const long long cost = rounds * (nt + 16);
        if (best < 0 || cost < best) { best = cost; c.nt = nt; c.tok_tiles = (int)tok_tiles; }
    }
    c.stage_bytes = MAT_BLOCK + c.nt / 2 * 128;
    c.tmem_cols = 2 * MAT_BULK_TOKENS;
    c.grid = 2u * (unsigned)std::min(ch_pairs * c.tok_tiles, pairs);
    stages_of(c, MAT_ROOM, MAT_STAGES_MAX);
    return c;
}

MatChoice choose(const imat_plan_t *p, long long rows)
{
    if ((long long)p->ch_tiles * ((rows + 127) / 128) <= 2 * p->sms) return choose_few(p, rows);
    return choose_bulk(p, rows);
}

int mat_opt_in(int *sms)
{
    static std::atomic<int> done[MAX_DEVICES];
    const int rc = umma_init_once();
    if (rc != ICONV_OK) return rc;
    const int dev = current_device_slot();
    if (dev < 0) { set_error("imat: no current device, or its index is beyond %d", MAX_DEVICES - 1); return ICONV_ERR_UNSUPPORTED; }
    if (!done[dev].load(std::memory_order_acquire)) {
        ICONV_CUDA_TRY(mat_opt_in_0());
        ICONV_CUDA_TRY(mat_opt_in_1());
        ICONV_CUDA_TRY(mat_opt_in_2());
        done[dev].store(1, std::memory_order_release);
    }
    *sms = umma_device_ready(dev);
    return ICONV_OK;
}

int build_plan(const imat_desc &d, cudaStream_t stream, imat_plan_t *p)
{
    p->n = d.n; p->k = d.k; p->out_dtype = d.out_dtype; p->act = d.act; p->gated = d.up_weights != nullptr;
    p->ch_tiles = p->gated ? (d.n + 63) / 64 : (d.n + 127) / 128;
    p->k_blocks = (d.k + 127) / 128;
    int rc = mat_opt_in(&p->sms);
    if (rc != ICONV_OK) return rc;
    p->device = current_device_slot();
    const size_t bytes = (size_t)p->ch_tiles * p->k_blocks * MAT_BLOCK;
    ICONV_CUDA_TRY(cudaMalloc((void **)&p->packed, bytes));
    ICONV_CUDA_TRY(cudaMalloc((void **)&p->row_params, (size_t)p->ch_tiles * BLOCK_M * sizeof(float2)));
    rc = umma_encode_2d(&p->tmap_w, p->packed, 128, (long long)(bytes / 128), 128, 128, BLOCK_M, 128);
    if (rc != ICONV_OK) return rc;
    PackArgs a;
    a.w[0] = d.weights; a.w[1] = d.up_weights; a.scales[0] = d.scales; a.scales[1] = d.up_scales; a.bias[0] = d.bias; a.bias[1] = d.up_bias;
    a.w_stride = d.w_stride; a.n = d.n; a.k = d.k; a.gated = p->gated; a.k_blocks = p->k_blocks;
    a.whole = !(((uintptr_t)d.weights | (uintptr_t)d.up_weights | (uintptr_t)d.w_stride) % 16);
    a.units = (long long)(bytes / 16); a.rows = p->ch_tiles * BLOCK_M;
    a.packed = (uint4 *)p->packed; a.row_params = p->row_params;
    const unsigned blocks = (unsigned)std::min<long long>((a.units + 255) / 256, 16ll * p->sms);
    mat_pack_kernel<<<blocks, 256, 0, stream>>>(a);
    ICONV_CUDA_TRY(cudaGetLastError());
    ICONV_CUDA_TRY(cudaStreamSynchronize(stream));
    return ICONV_OK;
}

int element(int dtype) { return dtype == ICONV_F32 ? 4 : 2; }

}  // namespace

}  // namespace iconv

using namespace iconv;

extern "C" int imat_plan_destroy(imat_plan_t *p)
{
    if (!p) return ICONV_OK;
    cudaFree(p->packed);
    cudaFree(p->row_params);
    delete p;
    return ICONV_OK;
}

extern "C" int imat_plan(const imat_desc *desc, void *cuda_stream, imat_plan_t **plan_out)
{
    if (!desc || !plan_out) { set_error("imat_plan: null argument"); return ICONV_ERR_ARG; }
    *plan_out = nullptr;
    const imat_desc &d = *desc;
    if (d.n < 1 || d.k < 1) { set_error("imat_plan: n and k must be positive"); return ICONV_ERR_ARG; }
    if (d.out_dtype != ICONV_F32 && d.out_dtype != ICONV_F16 && d.out_dtype != ICONV_BF16) { set_error("imat_plan: out_dtype must be F32, F16 or BF16"); return ICONV_ERR_ARG; }
    if (d.act < IMAT_NONE || d.act > IMAT_GELU_TANH) { set_error("imat_plan: bad activation"); return ICONV_ERR_ARG; }
    if (!d.weights || !d.scales) { set_error("imat_plan: weights and scales must be given"); return ICONV_ERR_ARG; }
    if (d.up_weights ? !d.up_scales : (d.up_scales || d.up_bias)) { set_error("imat_plan: up_weights and up_scales belong together, and up_bias to them"); return ICONV_ERR_ARG; }
    if (d.w_stride < d.k) { set_error("imat_plan: w_stride is shorter than a row"); return ICONV_ERR_SHAPE; }
    if (d.k > MAT_K_MAX) { set_error("imat_plan: sums over k = %d do not fit int32", d.k); return ICONV_ERR_OVERFLOW; }
    if ((uintptr_t)d.scales % 4 || (uintptr_t)d.bias % 4 || (uintptr_t)d.up_scales % 4 || (uintptr_t)d.up_bias % 4) {
        set_error("imat_plan: scales and biases must be 4-byte aligned");
        return ICONV_ERR_ALIGN;
    }
    if (d.n > (1 << 24) || (long long)d.n * d.k > (1ll << 37)) { set_error("imat_plan: weights too large"); return ICONV_ERR_SHAPE; }
    imat_plan_t *p = new (std::nothrow) imat_plan_s();
    if (!p) { set_error("imat_plan: out of host memory"); return ICONV_ERR_ARG; }
    const int rc = build_plan(d, (cudaStream_t)cuda_stream, p);
    if (rc != ICONV_OK) {
        imat_plan_destroy(p);
        return rc;
    }
    *plan_out = p;
    return ICONV_OK;
}

extern "C" int imat_plan_describe(const imat_plan_t *p, int64_t rows, char *text, size_t size)
{
    if (!p || !text || size == 0 || rows < 1 || rows > (1 << 30)) { set_error("imat_plan_describe: null argument or rows outside 1 ... 2^30"); return ICONV_ERR_ARG; }
    const MatChoice c = choose(p, rows);
    snprintf(text, size, "%s: tiles of %d channels x %d tokens, %u CTAs, split %d, %d stages of %d bytes%s", c.split ? "few" : "bulk", c.split ? 128 : 256, c.nt,
             c.grid, c.split ? c.split : 1, c.stages, c.stage_bytes, p->gated ? ", gated" : "");
    return ICONV_OK;
}

extern "C" int imat_forward(const imat_plan_t *p, int64_t rows, const int8_t *x, int64_t x_stride, const float *x_scales, const void *residual,
                            int64_t residual_stride, void *out, int64_t out_stride, void *cuda_stream)
{
    if (!p) { set_error("imat_forward: null plan"); return ICONV_ERR_ARG; }
    if (rows < 0 || rows > (1 << 30)) { set_error("imat_forward: rows must lie in 0 ... 2^30"); return ICONV_ERR_ARG; }
    if (x_stride < p->k || out_stride < p->n || (residual && residual_stride < p->n)) { set_error("imat_forward: a row stride is shorter than the row"); return ICONV_ERR_SHAPE; }
    if (residual && p->gated) { set_error("imat_forward: a gated product takes no residual"); return ICONV_ERR_UNSUPPORTED; }
    const long long most = 1ll << 40;               // bytes, or elements, of a matrix at most
    if (rows > 0 && (x_stride > most / rows || out_stride > most / rows || (residual && residual_stride > most / rows))) { set_error("imat_forward: matrix too large"); return ICONV_ERR_SHAPE; }
    if (rows == 0) return ICONV_OK;
    if (!x || !x_scales || !out) { set_error("imat_forward: x, x_scales and out must be given"); return ICONV_ERR_ARG; }
    if ((uintptr_t)x % 16 || x_stride % 16 || (uintptr_t)x_scales % 16) { set_error("imat_forward: x and x_scales must be 16-byte aligned, x_stride a multiple of 16"); return ICONV_ERR_ALIGN; }
    if (((uintptr_t)out | (uintptr_t)residual) % element(p->out_dtype)) { set_error("imat_forward: out and residual must be aligned to their element"); return ICONV_ERR_ALIGN; }
    if (current_device_slot() != p->device) { set_error("imat_forward: the plan belongs to device %d, which is not current", p->device); return ICONV_ERR_ARG; }
    const MatChoice c = choose(p, rows);
    const int box = c.split ? c.nt : c.nt / 2;
    CUtensorMap tmap_x;
    const int rc = umma_encode_2d(&tmap_x, x, p->k, rows, x_stride, 128, box, 128);
    if (rc != ICONV_OK) return rc;
    MatArgs a;
    memset(&a, 0, sizeof(a));
    a.m = rows; a.n = p->n;
    a.ch_tiles = p->ch_tiles; a.tok_tiles = c.tok_tiles; a.nt = c.nt; a.k_blocks = p->k_blocks;
    a.stages = c.stages; a.stage_bytes = c.stage_bytes; a.tmem_cols = c.tmem_cols;
    // D = s32, A = s8, B = s8, both K-major, N / 8, M / 16 (a pair's instruction spans both CTAs' channels)
    a.idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((unsigned)(c.nt >> 3) << 17) | ((unsigned)((c.split ? BLOCK_M : 2 * BLOCK_M) >> 4) << 24);
    a.act = p->act;
    a.row_params = p->row_params;
    a.x_scales = x_scales;
    a.residual = residual; a.ld_res = residual_stride;
    a.out = out; a.ld_out = out_stride;
    a.status = device_status_ptr();
    if (!a.status) { set_error("device status word not available"); return ICONV_ERR_CUDA; }
    const MatLaunch l = {c.grid, c.smem, (cudaStream_t)cuda_stream, c.split, &p->tmap_w, &tmap_x, &a};
    const bool gated = p->gated != 0;
    ICONV_CUDA_TRY((p->out_dtype == ICONV_F32 ? mat_launch_0(gated, l) : p->out_dtype == ICONV_F16 ? mat_launch_1(gated, l) : mat_launch_2(gated, l)));
    return ICONV_OK;
}
