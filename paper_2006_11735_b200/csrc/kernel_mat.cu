// Host side of the products of 8-bit rows with int8 weights (mat_device.cuh): validation, the plan's weight layout, which kernel and tile a
// call runs, the launch.
#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>

#include "mat_inst.h"

struct imat_plan_s {
    int n = 0, k = 0, out_dtype = 0, act = 0, gated = 0, device = -1, sms = 0;
    int ch_tiles = 0, k_blocks = 0;
    int8_t *packed = nullptr;              // [ch_tiles][k_blocks][128 rows][128 bytes]
    float2 *row_params = nullptr;          // behind them: [ch_tiles * 128] scale, bias
    CUtensorMap tmap_w;
};

namespace iconv {

namespace {

constexpr int MAT_K_MAX = 131071;          // 128 * 128 * k stays under 2^31

// What one call runs.
struct MatChoice {
    bool streams, bulk;                    // the streaming kernel, the bulk kernel, else the few-tile kernel
    int warps;                             // of a block of the streaming kernel
    int split;                             // parts of a tile's reduction
    int nt, tok_tiles, stages, stage_bytes, recv_bytes, tmem_cols;
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

constexpr int MAT_ROOM = MAX_SMEM - 1024 - (int)sizeof(MatShared);
constexpr int MAT_ROOM_HALF = MAX_SMEM / 2 - 1024 - 1024 - (int)sizeof(MatShared);      // two blocks on an SM (each takes 1 KB of the system's besides)

// Everything of a choice that follows from kernel, split and tokens of a tile.
MatChoice choice(const imat_plan_t *p, long long rows, bool bulk, int split, int nt)
{
    MatChoice c;
    c.streams = false; c.warps = 0;
    c.bulk = bulk; c.split = split; c.nt = nt;
    c.tok_tiles = (int)((rows + nt - 1) / nt);
    c.stage_bytes = MAT_BLOCK + (bulk ? nt / 2 : nt) * 128;
    c.recv_bytes = split > 1 ? (split - 1) * ((nt / MAT_PIECE + split - 1) / split) * MAT_PIECE_BYTES : 0;
    c.tmem_cols = bulk ? 2 * MAT_BULK_TOKENS : 32;
    while (c.tmem_cols < nt) c.tmem_cols *= 2;
    const long long tiles = (long long)(bulk ? (p->ch_tiles + 1) / 2 : p->ch_tiles) * c.tok_tiles;
    c.grid = bulk ? 2u * (unsigned)std::min<long long>(tiles, p->sms / 2) : (unsigned)(tiles * split);
    const int blocks = bulk ? MAT_STAGES_MAX : (p->k_blocks + split - 1) / split;
    const int room = bulk || c.grid <= (unsigned)p->sms ? MAT_ROOM : MAT_ROOM_HALF;
    c.stages = std::max(2, std::min(std::min((room - c.recv_bytes) / c.stage_bytes, MAT_STAGES_MAX), blocks));
    c.smem = 1024 + (size_t)c.stages * c.stage_bytes + c.recv_bytes + sizeof(MatShared);
    return c;
}

// Few tiles take sixteen warps each to keep the memory busy, many take four, several of them on an SM.
MatChoice choice_stream(const imat_plan_t *p, long long rows)
{
    MatChoice c = {};
    c.streams = true;
    const int blocks = p->gated ? (p->n + 15) / 16 : (p->n + 31) / 32, warps = blocks <= p->sms ? 16 : blocks <= 2 * p->sms ? 8 : 4;
    c.warps = warps; c.split = 1;
    c.nt = (int)rows; c.tok_tiles = 1;
    c.grid = (unsigned)(p->gated ? (p->n + 15) / 16 : (p->n + 31) / 32);
    c.smem = (size_t)warps * (rows > 8 ? 16 : 8) * MAT_STREAM_PITCH * 4;
    return c;
}

// Which kernel, tile and split a call runs: the least of a time estimate over what there is.  The estimate is in nanoseconds and follows what bounds each
// form on a B200 as measured: a block's way from L2 (87 bytes a nanosecond and SM, whatever the tile), its loads' latency (1100 ns for a round of
// its stages), the issue of its instructions (190 ns for a block of 128 bytes of the reduction), HBM, then the epilogue.  It only has to rank the forms: over
// 110 drawn sizes its choice took 3 % longer than the best of all forms on average (geometric mean), 33 % at most.
constexpr double SM_RATE = 87.0, HBM_RATE = 6300.0, ROUND_LATENCY = 1100.0, ISSUE = 190.0;

// Up to here a few tokens stream.  The streaming kernel's blocks fill the SM's registers, so that nothing of the kernel behind comes up beside them.  Whole sublayers of one
// token, 4096 wide, whose second product has 12 / 17 / 20 / 24 / 28 / 34 / 64 MB of weights: 13.0 / 16.3 / 18.5 / 21.3 / 22.7 / 26.5 / 42.3 us with it on this kernel, 13.4 / 17.3 /
// 18.8 / 20.8 / 22.0 / 24.8 / 40.3 on the few-tile kernel; of sixteen tokens 14.0 / 17.5 / 19.9 / 22.8 / 24.3 / 28.3 / 46.0 and 15.4 / 18.6 / 19.9 / 22.0 / 23.3 / 25.8 / 41.4.
constexpr double MAT_STREAM_BYTES = 24.0 * 1048576.0;

struct CallShape {
    long long rows;
    double weight_bytes, hbm;              // bytes of weights; nanoseconds that the call's bytes take from HBM
    int residual, act;
};

CallShape shape_of(const imat_plan_t *p, long long rows, bool residual)
{
    CallShape s;
    s.rows = rows;
    s.weight_bytes = (double)p->n * p->k * (p->gated ? 2 : 1);
    s.hbm = (s.weight_bytes + (double)rows * p->k + (double)rows * p->n * (p->out_dtype == ICONV_F32 ? 4 : 2) * (residual ? 2 : 1)) / HBM_RATE;
    s.residual = residual; s.act = p->act != IMAT_NONE && p->act != IMAT_RELU;
    return s;
}

// Few tokens, weights in registers: HBM at a rate that the tokens' own loads lower, or what an SM takes in.
double cost_stream(const imat_plan_t *p, const CallShape &s, const MatChoice &c)
{
    const double from_hbm = s.weight_bytes / (5900.0 - 47.0 * (double)(s.rows - 1));
    const double per_sm = (double)((c.grid + p->sms - 1) / p->sms) * MAT_STREAM_ROWS * 128.0 * p->k_blocks / (92.0 - 1.3 * (double)s.rows);
    return 1400.0 + std::max(from_hbm, per_sm) + 60.0 * (double)((s.rows + c.warps - 1) / c.warps);
}

// One tile per cluster.
double cost_few(const imat_plan_t *p, const CallShape &s, const MatChoice &c)
{
    const int kb = (p->k_blocks + c.split - 1) / c.split;
    const bool two = c.smem <= (size_t)MAX_SMEM / 2 - 1024;
    double at_once = (double)p->sms * (two ? 2 : 1);
    if (c.split == 8 && !two) at_once = 0.75 * p->sms;         // (so many large blocks are seldom free within one part of the chip)
    const double waves = std::max(1.0, std::ceil((double)c.grid / at_once));
    const double per_sm = c.grid <= (unsigned)p->sms ? 1.0 : 0.5 * ((double)c.grid / p->sms + std::ceil((double)c.grid / p->sms));
    const double load = std::max(per_sm * kb * c.stage_bytes / SM_RATE, waves * kb * ROUND_LATENCY / c.stages);
    const double groups = std::ceil((double)std::min<long long>(c.nt, s.rows) / 16.0);
    const double group = (p->gated ? 200.0 : 270.0) + 80.0 * s.act + 120.0 * s.residual;
    const double epilogue = c.split == 1 ? groups * group : 700.0 + std::ceil(c.nt / 32.0) * 250.0 + std::ceil((double)c.nt / (16 * c.split)) * (group + 100.0);
    return 1900.0 + (c.split > 1 ? 50.0 + 150.0 * c.split : 0.0) + std::max(std::max(load, waves * kb * ISSUE), s.hbm) + waves * epilogue + (waves - 1.0) * 1200.0;
}

// Persistent pairs: rounds of tiles, each bound by its sums or by the epilogue of the one before.
double cost_bulk(const imat_plan_t *p, const CallShape &s, const MatChoice &c)
{
    const double tiles = (double)((p->ch_tiles + 1) / 2) * c.tok_tiles, rounds = std::ceil(tiles / (p->sms / 2));
    const double sums = p->k_blocks * std::max((double)c.stage_bytes / SM_RATE, ISSUE);
    const double epilogue = 1100.0 + c.nt / 64.0 * ((p->gated ? 560.0 : 600.0) + 500.0 * s.residual + 100.0 * s.act);
    return std::max(2300.0 + sums + (rounds - 1.0) * std::max(sums, epilogue) + epilogue, 2300.0 + s.hbm);
}

MatChoice choose(const imat_plan_t *p, long long rows, bool residual)
{
    const CallShape s = shape_of(p, rows, residual);
    MatChoice best = {};
    double least = -1.0;
    auto offer = [&](const MatChoice &c, double cost) {
        if (c.smem <= (size_t)MAX_SMEM && (least < 0.0 || cost < least)) { least = cost; best = c; }
    };
    if (rows <= MAT_STREAM_TOKENS && s.weight_bytes <= MAT_STREAM_BYTES) {
        const MatChoice c = choice_stream(p, rows);
        offer(c, cost_stream(p, s, c));
    }
    const long long tiles16 = (long long)p->ch_tiles * ((rows + 15) / 16);
    for (int split = 1; split <= 8 && split <= p->k_blocks; split *= 2)
        for (int nt : {16, 32, 48, 64, 96, 128}) {
            if (nt >= rows + 16 && nt > 16) break;                 // the first that takes all rows is the last
            if (tiles16 * 16 / nt * split > 8ll * p->sms) continue;
            const MatChoice c = choice(p, rows, false, split, nt);
            offer(c, cost_few(p, s, c));
        }
    for (int nt = 64; nt <= 256; nt += 32) {
        const MatChoice c = choice(p, rows, true, 1, nt);
        offer(c, cost_bulk(p, s, c));
    }
    return best;
}

int mat_opt_in(int *sms)
{
    static std::atomic<int> done[MAX_DEVICES];
    const int rc = umma_init_once();
    if (rc != ICONV_OK) return rc;
    const int dev = current_device_slot();
    if (dev < 0) { set_error("imat: no current device, or its index is beyond %d", MAX_DEVICES - 1); return ICONV_ERR_UNSUPPORTED; }
    if (!done[dev].load(std::memory_order_acquire)) {
        ICONV_CUDA_TRY(mat_opt_in_0());        // (shared memory beyond 48 KB; it also has every instance loaded before a call may be captured)
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
    ICONV_CUDA_TRY(cudaMalloc((void **)&p->packed, bytes + (size_t)p->ch_tiles * BLOCK_M * sizeof(float2)));
    p->row_params = (float2 *)(p->packed + bytes);
    rc = umma_encode_2d(&p->tmap_w, p->packed, 128, (long long)(bytes / 128), 128, 128, BLOCK_M, 128);
    if (rc != ICONV_OK) return rc;
    PackArgs a;
    a.w[0] = d.weights; a.w[1] = d.up_weights; a.scales[0] = d.scales; a.scales[1] = d.up_scales; a.bias[0] = d.bias; a.bias[1] = d.up_bias;
    a.w_stride = d.w_stride; a.n = d.n; a.k = d.k; a.gated = p->gated; a.k_blocks = p->k_blocks;
    a.whole = !(((uintptr_t)d.weights | (uintptr_t)d.up_weights | (uintptr_t)d.w_stride) % 16);
    a.units = (long long)(bytes / 16); a.rows = p->ch_tiles * BLOCK_M;
    a.packed = (uint4 *)p->packed; a.row_params = p->row_params;
    const unsigned blocks = (unsigned)std::min<long long>((a.units + 255) / 256, 16ll * p->sms);
    const auto kernel = mat_pack_kernel;
    ICONV_CUDA_TRY(launch_kernel(kernel, false, blocks, 256, 0, stream, a));
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
    if (d.n > (1 << 24) || ((long long)d.n + 128) * (d.k + 127) * (d.up_weights ? 2 : 1) >= (1ll << 37)) { set_error("imat_plan: weights too large"); return ICONV_ERR_SHAPE; }
    if (d.w_stride > (1ll << 46) / d.n) { set_error("imat_plan: w_stride too large"); return ICONV_ERR_SHAPE; }
    // (an allocation or a wait would end a capture)
    cudaStreamCaptureStatus capture;
    ICONV_CUDA_TRY(cudaStreamIsCapturing((cudaStream_t)cuda_stream, &capture));
    if (capture != cudaStreamCaptureStatusNone) { set_error("imat_plan: the stream is capturing"); return ICONV_ERR_CUDA; }
    imat_plan_t *p = new (std::nothrow) imat_plan_s();
    if (!p) { set_error("imat_plan: out of host memory"); return ICONV_ERR_ARG; }
    const int rc = build_plan(d, (cudaStream_t)cuda_stream, p);
    if (rc != ICONV_OK) {
        imat_plan_destroy(p);
        cudaGetLastError();                // (an allocation that failed is reported here, not by whatever the caller launches next)
        return rc;
    }
    *plan_out = p;
    return ICONV_OK;
}

extern "C" int imat_plan_describe(const imat_plan_t *p, int64_t rows, char *text, size_t size)
{
    if (!p || !text || size == 0 || rows < 1 || rows > (1 << 30)) { set_error("imat_plan_describe: null argument or rows outside 1 ... 2^30"); return ICONV_ERR_ARG; }
    const MatChoice c = choose(p, rows, false);
    if (c.streams) snprintf(text, size, "stream: tiles of %d rows x %d tokens, %u blocks of %d warps%s", MAT_STREAM_ROWS, c.nt, c.grid, c.warps, p->gated ? ", gated" : "");
    else snprintf(text, size, "%s: tiles of %d channels x %d tokens, %u CTAs, split %d, %d stages of %d bytes%s", c.bulk ? "bulk" : "few", c.bulk ? 256 : 128,
             c.nt, c.grid, c.split, c.stages, c.stage_bytes, p->gated ? ", gated" : "");
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
    const MatChoice c = choose(p, rows, residual != nullptr);
    const int box = c.bulk ? c.nt / 2 : c.nt;
    CUtensorMap tmap_x;
    if (!c.streams) {
        const int rc = umma_encode_2d(&tmap_x, x, p->k, rows, x_stride, 128, box, 128);
        if (rc != ICONV_OK) return rc;
    }
    const MatStreamArgs s = {p->packed, x, x_stride, (p->k - 1) / 16 * 16};
    MatArgs a;
    memset(&a, 0, sizeof(a));
    a.m = rows; a.n = p->n;
    a.ch_tiles = p->ch_tiles; a.tok_tiles = c.tok_tiles; a.nt = c.nt; a.k_blocks = p->k_blocks;
    a.stages = c.stages; a.stage_bytes = c.stage_bytes; a.split = c.split; a.recv_bytes = c.recv_bytes; a.tmem_cols = c.tmem_cols;
    // D = s32, A = s8, B = s8, both K-major, N / 8, M / 16 (a pair's instruction spans both CTAs' channels)
    a.idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((unsigned)(c.nt >> 3) << 17) | ((unsigned)((c.bulk ? 2 * BLOCK_M : BLOCK_M) >> 4) << 24);
    a.act = p->act;
    a.row_params = p->row_params;
    a.x_scales = x_scales;
    a.residual = residual; a.ld_res = residual_stride;
    a.out = out; a.ld_out = out_stride;
    a.status = device_status_ptr();
    if (!a.status) { set_error("device status word not available"); return ICONV_ERR_CUDA; }
    const unsigned threads = c.streams ? 32u * (unsigned)c.warps : c.bulk ? MAT_BULK_THREADS : MAT_FEW_THREADS;
    const MatLaunch l = {c.grid, threads, c.smem, (cudaStream_t)cuda_stream, c.bulk, c.streams, &p->tmap_w, &tmap_x, &a, &s};
    const bool gated = p->gated != 0;
    ICONV_CUDA_TRY((p->out_dtype == ICONV_F32 ? mat_launch_0(gated, l) : p->out_dtype == ICONV_F16 ? mat_launch_1(gated, l) : mat_launch_2(gated, l)));
    return ICONV_OK;
}
