// The element-wise kernels of the feed-forward operators: bound by the bytes they move.
//   act_bwd  D = dY * act'(Z), gated D0 = dY * U * act'(G), D1 = dY * act(G), and the column sums of either (the gradients of the biases), taken
//            in fp32 before the rounding.  One read of each operand, one write of each result.
//   apply    Y = act(Z) + R, gated Y = act(G) * U, fp32
//   pack     a matrix as the tile kernel takes it: bfloat16, rows padded with zeros to whole 16-byte chunks
// A workgroup has a strip of 32 chunks of columns (16 bytes a lane, 512 a row) and eight rows at a time.  Column sums: a thread adds up its rows, the
// eight rows of threads meet in LDS, every workgroup writes one partial sum a column, and a second kernel adds these in a fixed order.
#include "ff.h"
#include "ff_act.h"

namespace {

constexpr int FFE_CH = 32, FFE_ROWS = 8;

struct ffe_args {
    int64_t rows;
    int cols, pcols;                  // results are written (zeros) up to pcols
    int act;
    ff_mat dY, Z0, Z1, D0, D1;
    float *partial;                   // [gridDim.y][1 or 2][cols] or null
};

template <int T, int V, bool GATED> __global__ __launch_bounds__(256) void ff_act_bwd_kernel(ffe_args a)
{
    __shared__ float red[FFE_ROWS][FFE_CH * V];
    const int tx = threadIdx.x % FFE_CH, ty = threadIdx.x / FFE_CH;
    const int col = (blockIdx.x * FFE_CH + tx) * V, left = a.cols - col;
    float s0[V], s1[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s0[i] = s1[i] = 0.f;
    if (col < a.pcols) {
        for (int64_t row = (int64_t)blockIdx.y * FFE_ROWS + ty; row < a.rows; row += (int64_t)gridDim.y * FFE_ROWS) {
            float dy[V], g[V], u[V], d0[V], d1[V];
            ff_load<T, V>(dy, a.dY, row, col, left);
            ff_load<T, V>(g, a.Z0, row, col, left);
            if (GATED) ff_load<T, V>(u, a.Z1, row, col, left);
            ff_with_act(a.act, [&](auto act) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const ff_act_pair p = ff_act_both<decltype(act)::value>(g[i]);
                    d0[i] = dy[i] * (GATED ? u[i] * p.d : p.d);
                    d1[i] = dy[i] * p.f;
                }
            });
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (i >= left) d0[i] = d1[i] = 0.f;
                s0[i] += d0[i];
                s1[i] += d1[i];
            }
            ff_store<T, V>(d0, a.D0, row, col, a.pcols - col);
            if (GATED) ff_store<T, V>(d1, a.D1, row, col, a.pcols - col);
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int q = 0; q < (GATED ? 2 : 1); ++q) {
        if (q) __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) red[ty][tx * V + i] = q ? s1[i] : s0[i];
        __syncthreads();
        const int j = threadIdx.x, c = blockIdx.x * FFE_CH * V + j;
        if (j < FFE_CH * V && c < a.cols) {
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < FFE_ROWS; ++w) t += red[w][j];
            a.partial[((int64_t)blockIdx.y * (GATED ? 2 : 1) + q) * a.cols + c] = t;
        }
    }
}

// out[which][col] = sum over the workgroups of partial[w][which][col], sixteen interleaved chains a column and then the chains in order
__global__ __launch_bounds__(1024) void ff_colsum_kernel(const float *__restrict__ partial, int n, int cols, int outs, float *__restrict__ o0, float *__restrict__ o1)
{
    __shared__ float red[1024];
    const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6, j = blockIdx.x * 64 + tx;
    float s = 0.f;
    if (j < outs * cols) {
#pragma unroll 8
        for (int w = ty; w < n; w += 16) s += partial[(int64_t)w * outs * cols + j];
    }
    red[threadIdx.x] = s;
    __syncthreads();
    if (ty == 0 && j < outs * cols) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) t += red[w * 64 + tx];
        float *o = j < cols ? o0 : o1;
        if (o) o[j < cols ? j : j - cols] = t;
    }
}

template <bool GATED> __global__ __launch_bounds__(256) void ff_apply_kernel(ffe_args a)
{
    constexpr int V = 4;
    const int col = (blockIdx.x * FFE_CH + threadIdx.x % FFE_CH) * V, left = a.cols - col;
    if (left <= 0) return;
    for (int64_t row = (int64_t)blockIdx.y * FFE_ROWS + threadIdx.x / FFE_CH; row < a.rows; row += (int64_t)gridDim.y * FFE_ROWS) {
        float g[V], u[V], y[V];
        ff_load<FF_T32, V>(g, a.Z0, row, col, left);
        if (a.Z1.p) ff_load<FF_T32, V>(u, a.Z1, row, col, left);
        ff_with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                y[i] = ff_act<decltype(act)::value>(g[i]);
                if (GATED) y[i] *= u[i];
                else if (a.Z1.p) y[i] += u[i];
            }
        });
        ff_store<FF_T32, V>(y, a.D0, row, col, left);
    }
}

template <int T> __global__ __launch_bounds__(256) void ff_pack_kernel(ff_mat src, int64_t rows, int cols, int pcols, ff_mat dst)
{
    const int chunks = pcols / 8;
    const int64_t n = rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / chunks;
        const int col = 8 * (int)(i % chunks);
        float v[8];
        ff_load<T, 8>(v, src, row, col, cols - col);
        ff_store<FF_T16, 8>(v, dst, row, col, 8);
    }
}

__global__ __launch_bounds__(256) void ff_copy32_kernel(ff_mat src, int64_t rows, int cols, int pcols, ff_mat dst)
{
    const int chunks = (pcols + 3) / 4;
    const int64_t n = rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / chunks;
        const int col = 4 * (int)(i % chunks);
        float v[4];
        ff_load<FF_T32, 4>(v, src, row, col, cols - col);
        ff_store<FF_T32, 4>(v, dst, row, col, pcols - col);
    }
}

__global__ __launch_bounds__(256) void ff_zero_kernel(ff_mat m, int64_t rows, int64_t cols)
{
    const int64_t n = rows * cols;
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) ff_store<FF_TANY, 4>(zero, m, i / cols, i % cols, 1);
}

// workgroups along the rows: enough to fill the chip, few enough for the column sums
unsigned row_blocks(int64_t rows, unsigned strips) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(cdiv(rows, FFE_ROWS), std::max(1u, 2048 / strips))); }

unsigned flat_blocks(int64_t n) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(cdiv(n, 256), 1 << 16)); }

} // namespace

size_t sgnn_ff_sums_ws_bytes(uint64_t cols)
{
    // one partial sum a column, projection and workgroup along the rows: 2048 workgroups in all, or one for every strip of 128 columns
    return 2 * 4 * std::max<uint64_t>(2048 * 256, cols) + 4 * 4 * cols + 512;
}

int sgnn_launch_ff_act_bwd(sgnn_ctx *ctx, int64_t rows, int64_t cols, int64_t pcols, int act, const ff_mat &dY, const ff_mat &Z0, const ff_mat *Z1,
                           const ff_mat &D0, const ff_mat *D1, float *const *db, ws_alloc *ws, hipStream_t st)
{
    ffe_args a = {};
    a.rows = rows; a.cols = (int)cols; a.pcols = (int)pcols; a.act = act;
    a.dY = dY; a.Z0 = Z0; a.D0 = D0;
    if (Z1) { a.Z1 = *Z1; a.D1 = *D1; }
    const bool all16 = dY.b16 && Z0.b16 && (!Z1 || Z1->b16) && D0.b16, all32 = !dY.b16 && !Z0.b16 && (!Z1 || !Z1->b16) && !D0.b16;
    const int v = all32 ? 4 : 8, outs = Z1 ? 2 : 1;
    const unsigned strips = cdiv(pcols, FFE_CH * v), blocks = row_blocks(rows, strips);
    const bool sums = db[0] || (Z1 && db[1]);
    const size_t off = ws->off;
    if (sums) {
        a.partial = ws->get<float>((size_t)blocks * outs * cols);
        if (!ws->ok) return sgnn_fail(ctx, SGNN_ERR_CAPACITY, "feed-forward operator: scratch too small: call sgnn_ctx_reserve_ffn");
    }
    const dim3 grid(strips, blocks), block(256);
#define SGNN_FFE(T_, V_, G_) SGNN_LAUNCH(ctx, st, "ff_act_bwd_kernel", SGNN_TAG, (ff_act_bwd_kernel<T_, V_, G_>), grid, block, 0, st, a)
    if (Z1) {
        if (all16) SGNN_FFE(FF_T16, 8, true);
        else if (all32) SGNN_FFE(FF_T32, 4, true);
        else SGNN_FFE(FF_TANY, 8, true);
    } else {
        if (all16) SGNN_FFE(FF_T16, 8, false);
        else if (all32) SGNN_FFE(FF_T32, 4, false);
        else SGNN_FFE(FF_TANY, 8, false);
    }
#undef SGNN_FFE
    if (sums)
        SGNN_LAUNCH(ctx, st, "ff_colsum_kernel", SGNN_TAG, ff_colsum_kernel, dim3(cdiv(outs * cols, 64)), dim3(1024), 0, st, a.partial, (int)blocks, (int)cols,
                    outs, db[0], Z1 ? db[1] : nullptr);
    ws->off = off;
    return SGNN_OK;
}

int sgnn_launch_ff_apply(sgnn_ctx *ctx, int64_t rows, int64_t cols, int act, const ff_mat &Z0, const ff_mat *Z1, const ff_mat &R, const ff_mat &Y, hipStream_t st)
{
    ffe_args a = {};
    a.rows = rows; a.cols = (int)cols; a.act = act;
    a.Z0 = Z0; a.Z1 = Z1 ? *Z1 : R; a.D0 = Y;
    const unsigned strips = cdiv(cols, FFE_CH * 4);
    const dim3 grid(strips, row_blocks(rows, strips));
    if (Z1) SGNN_LAUNCH(ctx, st, "ff_apply_kernel", SGNN_TAG, ff_apply_kernel<true>, grid, dim3(256), 0, st, a);
    else SGNN_LAUNCH(ctx, st, "ff_apply_kernel", SGNN_TAG, ff_apply_kernel<false>, grid, dim3(256), 0, st, a);
    return SGNN_OK;
}

int sgnn_launch_ff_pack(sgnn_ctx *ctx, const ff_mat &src, int64_t rows, int64_t cols, u16 *dst, int64_t ldd, hipStream_t st)
{
    const int64_t pcols = ff_pad8(cols);
    const ff_mat d = {dst, ldd, 1};
    const dim3 grid(flat_blocks(rows * (pcols / 8)));
    if (src.b16) SGNN_LAUNCH(ctx, st, "ff_pack_kernel", SGNN_TAG, ff_pack_kernel<FF_T16>, grid, dim3(256), 0, st, src, rows, (int)cols, (int)pcols, d);
    else SGNN_LAUNCH(ctx, st, "ff_pack_kernel", SGNN_TAG, ff_pack_kernel<FF_T32>, grid, dim3(256), 0, st, src, rows, (int)cols, (int)pcols, d);
    return SGNN_OK;
}

int sgnn_launch_ff_copy32(sgnn_ctx *ctx, const float *src, int64_t lds_, int64_t rows, int64_t cols, int64_t pcols, float *dst, int64_t ldd, hipStream_t st)
{
    const ff_mat s = {src, lds_, 0}, d = {dst, ldd, 0};
    SGNN_LAUNCH(ctx, st, "ff_copy32_kernel", SGNN_TAG, ff_copy32_kernel, dim3(flat_blocks(rows * ((pcols + 3) / 4))), dim3(256), 0, st, s, rows, (int)cols, (int)pcols, d);
    return SGNN_OK;
}

int sgnn_launch_ff_zero(sgnn_ctx *ctx, const ff_mat &m, int64_t rows, int64_t cols, hipStream_t st)
{
    SGNN_LAUNCH(ctx, st, "ff_zero_kernel", SGNN_TAG, ff_zero_kernel, dim3(flat_blocks(rows * cols)), dim3(256), 0, st, m, rows, cols);
    return SGNN_OK;
}
