// The element-wise kernels of the feed-forward operators: bound by the bytes they move.
//   act_bwd  D = dY * act'(Z), gated D0 = dY * U * act'(G), D1 = dY * act(G), and the column sums of either (the gradients of the biases), taken
//            in fp32 before the rounding.  One read of each operand, one write of each result.
//   row_parts, parts   an fp32 matrix as two planes of fp16 parts, scaled by powers of two (ff_gemm.hip says how and why): by one for each row from the
//            row's largest magnitude, or by a given one
//   pack     a matrix as the tile kernel takes it: bfloat16, rows padded with zeros to whole 16-byte chunks
// A workgroup of act_bwd has a strip of CH chunks of columns (16 bytes a lane; 32 of them, or as few as hold a narrow matrix) and 256 / CH rows at a time.  Column
// sums: a thread adds up its rows, the rows of threads meet in LDS, every workgroup writes one partial sum a column, and a second kernel adds these in
// a fixed order.
#include "ff.h"
#include "ff_act.h"

namespace {

struct ffe_args {
    int64_t rows;
    int cols, pcols;                  // results are written (zeros) up to pcols
    int act;
    ff_mat dY, Z0, Z1, D0, D1;
    float *partial;                   // [gridDim.y][1 or 2][cols] or null
};

// Magnitudes are compared as the bits they have, which are in the same order (and tell the smallest ones from zero in every mode of the arithmetic).
__device__ __forceinline__ uint32_t finite_max(uint32_t m, float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
    return b < 0x7f800000u ? max(m, b) : m;
}

// The workgroup's largest m (of 256 threads), in thread 0
__device__ __forceinline__ uint32_t block_max(uint32_t m)
{
    __shared__ uint32_t red[4];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    return max(max(red[0], red[1]), max(red[2], red[3]));
}

template <int T, int V, bool GATED, int FFE_CH> __global__ __launch_bounds__(256) void ff_act_bwd_kernel(ffe_args a)
{
    constexpr int FFE_ROWS = 256 / FFE_CH;
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
            if (a.D0.p) ff_store<T, V>(d0, a.D0, row, col, a.pcols - col);
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
#pragma unroll 8
            for (int w = 0; w < FFE_ROWS; ++w) t += red[w][j];
            a.partial[((int64_t)blockIdx.y * (GATED ? 2 : 1) + q) * a.cols + c] = t;
        }
    }
}

// out[which][col] = sum over the workgroups of partial[w][which][col]: 64 interleaved chains a column, sixteen columns a workgroup, and then the chains in order
__global__ __launch_bounds__(1024) void ff_colsum_kernel(const float *__restrict__ partial, int n, int cols, int outs, float *__restrict__ o0, float *__restrict__ o1)
{
    __shared__ float red[1024];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, j = blockIdx.x * 16 + tx;
    float s = 0.f;
    if (j < outs * cols) {
#pragma unroll 8
        for (int w = ty; w < n; w += 64) s += partial[(int64_t)w * outs * cols + j];
    }
    red[threadIdx.x] = s;
    __syncthreads();
    if (ty == 0 && j < outs * cols) {
        float t = 0.f;
#pragma unroll 16
        for (int w = 0; w < 64; ++w) t += red[w * 16 + tx];
        float *o = j < cols ? o0 : o1;
        if (o) o[j < cols ? j : j - cols] = t;
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

__global__ __launch_bounds__(256) void ff_convert_kernel(ff_mat src, int64_t rows, int cols, ff_mat dst)
{
    const int chunks = (cols + 7) / 8;
    const int64_t n = rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / chunks;
        const int col = 8 * (int)(i % chunks);
        float v[8];
        ff_load<FF_TANY, 8>(v, src, row, col, cols - col);
        ff_store<FF_TANY, 8>(v, dst, row, col, cols - col);
    }
}

// f(row, first column) for the chunks of V columns of a matrix, dealt to the threads of `groups` workgroups
template <int V, class F> __device__ __forceinline__ void for_chunks(int64_t rows, int64_t cols, unsigned groups, F f)
{
    const int64_t chunks = (cols + V - 1) / V, n = rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)groups * 256) {
        const int64_t row = n <= 0xffffffffll ? (int64_t)((uint32_t)i / (uint32_t)chunks) : i / chunks;
        f(row, V * (i - row * chunks));
    }
}

__device__ __forceinline__ int exponent_of(uint32_t bits, int none) { return bits ? 14 + 127 - (int)(bits >> 23) : none; }

// eight values times 2^ex as their parts: the eight first ones, then the eight second ones
__device__ __forceinline__ void store_parts(const float (&v)[8], int ex, u16 *to)
{
    _Float16 h[2][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = __builtin_amdgcn_ldexpf(v[e], ex);
        h[0][e] = (_Float16)x;
        const float r = (x - (float)h[0][e]) * 2048.f;
        h[1][e] = (_Float16)(fabsf(x) < __builtin_inff() ? r : 0.f);
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) *reinterpret_cast<u32x4 *>(to + 8 * q) = *reinterpret_cast<const u32x4 *>(h[q]);
}

struct ffe_rows { ff_row_parts r; ff_scan w[2]; uint32_t *largest; int scans; };

// G lanes a row; CH chunks of eight values a lane stay in registers, or (CH = 0) a row is read once for its largest magnitude and once for its parts
template <int G, int CH> __global__ __launch_bounds__(256) void ff_row_parts_kernel(ffe_rows s, unsigned groups)
{
    if (blockIdx.y > 0) {
        if ((int)blockIdx.x >= s.scans) return;
        const ff_scan &m = s.w[blockIdx.y - 1];
        const ff_mat src = {m.p, m.ld, 0};
        uint32_t largest = 0;
        for_chunks<8>(m.rows, m.cols, s.scans, [&](int64_t row, int64_t col) {
            float v[8];
            ff_load<FF_T32, 8>(v, src, row, col, (int)min(m.cols - col, (int64_t)8));
#pragma unroll
            for (int e = 0; e < 8; ++e) largest = finite_max(largest, v[e]);
        });
        const uint32_t t = block_max(largest);
        if (threadIdx.x == 0) s.largest[(blockIdx.y - 1) * s.scans + blockIdx.x] = t;
        return;
    }
    if (blockIdx.x >= groups) return;
    const ff_row_parts &p = s.r;
    const ff_mat src = {p.m.p, p.m.ld, 0};
    const int l = threadIdx.x % G;
    const int64_t chunks = (p.m.cols + 7) / 8;
    int key = 0;
    for (int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G; row < p.m.rows; row += (int64_t)groups * (256 / G)) {
        float v[CH ? CH : 1][8];
        uint32_t largest = 0;
        auto each = [&](auto f) {
            if constexpr (CH > 0) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (c * G + l < chunks) f(v[c], (int64_t)8 * (c * G + l));
            } else
                for (int64_t c = l; c < chunks; c += G) f(v[0], 8 * c);
        };
        auto load = [&](float (&x)[8], int64_t col) { ff_load<FF_T32, 8>(x, src, row, col, (int)min(p.m.cols - col, (int64_t)8)); };
        if constexpr (CH > 0) each(load);          // all of them requested together
        each([&](float (&x)[8], int64_t col) {
            if constexpr (CH == 0) load(x, col);
#pragma unroll
            for (int e = 0; e < 8; ++e) largest = finite_max(largest, x[e]);
        });
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) largest = max(largest, (uint32_t)__shfl_xor((int)largest, o, 64));
        const int ex = exponent_of(largest, FF_EX_ZERO);
        if (l == 0) p.ex[row] = ex;
        if (p.other) key = max(key, FF_EX_KEY - ex - p.other[row]);
        if (p.to)
            each([&](float (&x)[8], int64_t col) {
                if constexpr (CH == 0) load(x, col);
                store_parts(x, ex, p.to + row * p.ld + 2 * col);
            });
    }
    if (p.key) {
        const uint32_t t = block_max((uint32_t)key);
        if (threadIdx.x == 0) p.key[blockIdx.x] = t;
    }
}

// act_bwd of fp32 matrices straight into parts: a row's gradients (of both projections) stay in the registers of its G lanes, CH chunks of eight columns a
// lane, until their largest magnitude is known.  What it saves is a write and a read of D.
template <bool GATED, int G, int CH> __global__ __launch_bounds__(256) void ff_act_bwd_parts_kernel(ffe_args a, ff_row_parts p)
{
    constexpr int RPW = 256 / G;
    __shared__ float red[RPW > 1 ? 256 * CH * 8 : 1];
    __shared__ uint32_t row_max[4];
    const int l = threadIdx.x % G, grp = threadIdx.x / G;
    float s0[CH][8], s1[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) s0[c][i] = s1[c][i] = 0.f;
    int key = 0;
    for (int64_t row = (int64_t)blockIdx.x * RPW + grp; row < a.rows; row += (int64_t)gridDim.x * RPW) {
        float d0[CH][8], d1[CH][8], u[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = 8 * (c * G + l), left = a.cols - col;
            // behind the last column every value is 0, and so are the gradients there
            ff_load<FF_T32, 8>(d0[c], a.dY, row, col, left);
            ff_load<FF_T32, 8>(d1[c], a.Z0, row, col, left);
            if (GATED) ff_load<FF_T32, 8>(u[c], a.Z1, row, col, left);
        }
        uint32_t largest = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            ff_with_act(a.act, [&](auto act) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const ff_act_pair f = ff_act_both<decltype(act)::value>(d1[c][i]);
                    const float dy = d0[c][i];
                    d0[c][i] = dy * (GATED ? u[c][i] * f.d : f.d);
                    d1[c][i] = dy * f.f;
                }
            });
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s0[c][i] += d0[c][i];
                largest = finite_max(largest, d0[c][i]);
                if (GATED) {
                    s1[c][i] += d1[c][i];
                    largest = finite_max(largest, d1[c][i]);
                }
            }
        }
#pragma unroll
        for (int o = (G < 64 ? G : 64) / 2; o > 0; o >>= 1) largest = max(largest, (uint32_t)__shfl_xor((int)largest, o, 64));
        if constexpr (G > 64) {
            // one row a workgroup: its wavefronts reach the barriers together
            __syncthreads();
            if ((threadIdx.x & 63) == 0) row_max[threadIdx.x >> 6] = largest;
            __syncthreads();
            largest = max(max(row_max[0], row_max[1]), max(row_max[2], row_max[3]));
        }
        const int ex = exponent_of(largest, FF_EX_ZERO);
        if (l == 0) p.ex[row] = ex;
        if (p.other) key = max(key, FF_EX_KEY - ex - p.other[row]);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = 8 * (c * G + l);
            if (col >= a.pcols) continue;
            store_parts(d0[c], ex, p.to + row * p.ld + 2 * col);
            if (GATED) store_parts(d1[c], ex, p.to + row * p.ld + 2 * (a.pcols + col));
        }
    }
    if (p.key) {
        const uint32_t t = block_max((uint32_t)key);
        if (threadIdx.x == 0) p.key[blockIdx.x] = t;
    }
    if (!a.partial) return;
#pragma unroll
    for (int q = 0; q < (GATED ? 2 : 1); ++q) {
        float *o = a.partial + ((int64_t)blockIdx.x * (GATED ? 2 : 1) + q) * a.cols;
        if constexpr (RPW == 1) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (8 * (c * G + l) + i < a.cols) o[8 * (c * G + l) + i] = q ? s1[c][i] : s0[c][i];
        } else {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) red[grp * (G * CH * 8) + 8 * (c * G + l) + i] = q ? s1[c][i] : s0[c][i];
            __syncthreads();
            for (int j = threadIdx.x; j < a.cols; j += 256) {
                float t = 0.f;
#pragma unroll
                for (int w = 0; w < RPW; ++w) t += red[w * (G * CH * 8) + j];
                o[j] = t;
            }
        }
    }
}

struct ffe_parts { ff_parts m[3]; };

__global__ __launch_bounds__(256) void ff_parts_kernel(ffe_parts s)
{
    const ff_parts &p = s.m[blockIdx.y];
    const ff_mat src = {p.m.p, p.m.ld, 0};
    uint32_t largest = 0;
    for (int i = threadIdx.x; i < p.words; i += 256) largest = max(largest, p.word[i]);
    largest = block_max(largest);
    const int ex = p.rows ? FF_EX_KEY - (int)largest : exponent_of(largest, 0);
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.ex = ex;
    for_chunks<8>(p.m.rows, p.m.cols, gridDim.x, [&](int64_t row, int64_t col) {
        float v[8];
        ff_load<FF_T32, 8>(v, src, row, col, (int)min(p.m.cols - col, (int64_t)8));
        store_parts(v, p.rows ? ex - p.rows[row] : ex, p.to + row * p.ld + 2 * col);
    });
}

__global__ __launch_bounds__(256) void ff_zero_kernel(ff_mat m, int64_t rows, int64_t cols)
{
    const int64_t n = rows * cols;
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) ff_store<FF_TANY, 4>(zero, m, i / cols, i % cols, 1);
}

unsigned flat_blocks(int64_t n) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(cdiv(n, 256), 1 << 16)); }

} // namespace

size_t sgnn_ff_sums_ws_bytes(uint64_t cols)
{
    // one partial sum a column, projection and workgroup along the rows: of these 2048 in all strips, or for every strip one; 2048 for rows of up to 4096
    return 2 * 4 * std::max<uint64_t>(std::max<uint64_t>(2048 * 256, cols), 2048 * std::min<uint64_t>(cols, 4096)) + 512;
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
    const int64_t chunks = cdiv(pcols, v);
    const unsigned ch = chunks <= 8 ? 8 : (chunks <= 16 ? 16 : 32), strips = cdiv(chunks, ch);
    // workgroups along the rows: enough to fill the chip, few enough for the column sums
    const unsigned blocks = (unsigned)std::max<int64_t>(1, std::min<int64_t>(cdiv(rows, 256 / ch), std::max(1u, 2048 / strips)));
    const bool sums = db[0] || (Z1 && db[1]);
    const size_t off = ws->off;
    if (sums) {
        a.partial = ws->get<float>((size_t)blocks * outs * cols);
        if (!ws->ok) return sgnn_fail(ctx, SGNN_ERR_CAPACITY, "feed-forward operator: scratch too small: call sgnn_ctx_reserve_ffn");
    }
    const dim3 grid(strips, blocks), block(256);
#define SGNN_FFE_CH(T_, V_, G_, CH_) SGNN_LAUNCH(ctx, st, "ff_act_bwd_kernel", SGNN_TAG, (ff_act_bwd_kernel<T_, V_, G_, CH_>), grid, block, 0, st, a)
#define SGNN_FFE(T_, V_, G_)                             \
    do {                                                 \
        if (ch == 8) SGNN_FFE_CH(T_, V_, G_, 8);         \
        else if (ch == 16) SGNN_FFE_CH(T_, V_, G_, 16);  \
        else SGNN_FFE_CH(T_, V_, G_, 32);                \
    } while (0)
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
#undef SGNN_FFE_CH
    if (sums)
        SGNN_LAUNCH(ctx, st, "ff_colsum_kernel", SGNN_TAG, ff_colsum_kernel, dim3(cdiv(outs * cols, 16)), dim3(1024), 0, st, a.partial, (int)blocks, (int)cols,
                    outs, db[0], Z1 ? db[1] : nullptr);
    ws->off = off;
    return SGNN_OK;
}

// workgroups along the rows of act_bwd_parts, each with a word of key and a partial sum a column: 0 where the rows are too wide for it
unsigned sgnn_ff_act_bwd_parts_groups(int64_t rows, int64_t pcols)
{
    const int64_t chunks = pcols / 8, per = chunks <= 16 ? 16 : (chunks <= 32 ? 8 : (chunks <= 128 ? 4 : 1));
    return chunks > 512 ? 0 : (unsigned)std::max<int64_t>(1, std::min<int64_t>(cdiv(rows, per), 2048));
}

int sgnn_launch_ff_act_bwd_parts(sgnn_ctx *ctx, int64_t rows, int64_t cols, int64_t pcols, int act, const ff_mat &dY, const ff_mat &Z0, const ff_mat *Z1,
                                 const ff_row_parts &p, float *const *db, ws_alloc *ws, hipStream_t st)
{
    ffe_args a = {};
    a.rows = rows; a.cols = (int)cols; a.pcols = (int)pcols; a.act = act;
    a.dY = dY; a.Z0 = Z0;
    if (Z1) a.Z1 = *Z1;
    const int outs = Z1 ? 2 : 1;
    const unsigned groups = sgnn_ff_act_bwd_parts_groups(rows, pcols);
    const bool sums = db[0] || (Z1 && db[1]);
    const size_t off = ws->off;
    if (sums) {
        a.partial = ws->get<float>((size_t)groups * outs * cols);
        if (!ws->ok) return sgnn_fail(ctx, SGNN_ERR_CAPACITY, "feed-forward operator: scratch too small: call sgnn_ctx_reserve_ffn");
    }
    auto run = [&](auto g, auto ch) -> int {
        constexpr int G = decltype(g)::value, CH = decltype(ch)::value;
        if (Z1) SGNN_LAUNCH(ctx, st, "ff_act_bwd_parts_kernel", SGNN_TAG, (ff_act_bwd_parts_kernel<true, G, CH>), dim3(groups), dim3(256), 0, st, a, p);
        else SGNN_LAUNCH(ctx, st, "ff_act_bwd_parts_kernel", SGNN_TAG, (ff_act_bwd_parts_kernel<false, G, CH>), dim3(groups), dim3(256), 0, st, a, p);
        return SGNN_OK;
    };
    const int64_t chunks = pcols / 8;
    using std::integral_constant;
    const int rc = chunks <= 16 ? run(integral_constant<int, 16>(), integral_constant<int, 1>()) : chunks <= 32 ? run(integral_constant<int, 32>(), integral_constant<int, 1>())
                 : chunks <= 64 ? run(integral_constant<int, 64>(), integral_constant<int, 1>()) : chunks <= 128 ? run(integral_constant<int, 64>(), integral_constant<int, 2>())
                 : chunks <= 256 ? run(integral_constant<int, 256>(), integral_constant<int, 1>()) : run(integral_constant<int, 256>(), integral_constant<int, 2>());
    if (rc) return rc;
    if (sums)
        SGNN_LAUNCH(ctx, st, "ff_colsum_kernel", SGNN_TAG, ff_colsum_kernel, dim3(cdiv(outs * cols, 16)), dim3(1024), 0, st, a.partial, (int)groups, (int)cols, outs,
                    db[0], Z1 ? db[1] : nullptr);
    ws->off = off;
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

int sgnn_launch_ff_convert(sgnn_ctx *ctx, const ff_mat &src, int64_t rows, int64_t cols, const ff_mat &dst, hipStream_t st)
{
    SGNN_LAUNCH(ctx, st, "ff_convert_kernel", SGNN_TAG, ff_convert_kernel, dim3(flat_blocks(rows * ((cols + 7) / 8))), dim3(256), 0, st, src, rows, (int)cols, dst);
    return SGNN_OK;
}

// workgroups of a launch: one for every 256 / G rows up to as many as may leave a word each
unsigned sgnn_ff_row_groups(int64_t rows, int64_t cols)
{
    const int64_t chunks = cdiv(cols, 8), per = chunks <= 16 ? 16 : (chunks <= 32 ? 8 : 4);
    return (unsigned)std::min<int64_t>(std::max<int64_t>(cdiv(rows, per), 1), FF_ROW_WORDS);
}

unsigned sgnn_ff_scan_groups(int n, const ff_scan *w)
{
    int64_t most = 1;
    for (int i = 0; i < n; ++i) most = std::max<int64_t>(most, w[i].rows * w[i].cols);
    return (unsigned)std::min<int64_t>(cdiv(most, 256 * 8), FF_SCAN_WORDS);
}

int sgnn_launch_ff_row_parts(sgnn_ctx *ctx, const ff_row_parts &r, int n, const ff_scan *w, uint32_t *largest, hipStream_t st)
{
    ffe_rows s = {};
    s.r = r;
    s.largest = largest;
    for (int i = 0; i < n; ++i) s.w[i] = w[i];
    s.scans = n ? (int)sgnn_ff_scan_groups(n, w) : 0;
    const int64_t chunks = cdiv(r.m.cols, 8);
    auto run = [&](auto g, auto ch) -> int {
        constexpr int G = decltype(g)::value, CH = decltype(ch)::value;
        const unsigned rows = sgnn_ff_row_groups(r.m.rows, r.m.cols);
        // the workgroups of y = 0 beyond those of the rows find none (and would leave words nobody counts)
        SGNN_LAUNCH(ctx, st, "ff_row_parts_kernel", SGNN_TAG, (ff_row_parts_kernel<G, CH>), dim3(std::max(rows, (unsigned)s.scans), 1 + n), dim3(256), 0, st, s, rows);
        return SGNN_OK;
    };
    // the fewest lanes that hold a row, one chunk each up to a wavefront
    if (chunks <= 16) return run(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    if (chunks <= 32) return run(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
    if (chunks <= 64) return run(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    if (chunks <= 128) return run(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    if (chunks <= 256) return run(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
    return run(std::integral_constant<int, 64>(), std::integral_constant<int, 0>());
}

int sgnn_launch_ff_parts(sgnn_ctx *ctx, int n, const ff_parts *m, hipStream_t st)
{
    ffe_parts s = {};
    int64_t most = 0;
    for (int i = 0; i < n; ++i) {
        s.m[i] = m[i];
        most = std::max(most, m[i].m.rows * (m[i].m.cols + 7));
    }
    const unsigned blocks = (unsigned)std::max<int64_t>(1, std::min<int64_t>(cdiv(most, 256 * 8), 4096));
    SGNN_LAUNCH(ctx, st, "ff_parts_kernel", SGNN_TAG, ff_parts_kernel, dim3(blocks, n), dim3(256), 0, st, s);
    return SGNN_OK;
}

int sgnn_launch_ff_zero(sgnn_ctx *ctx, const ff_mat &m, int64_t rows, int64_t cols, hipStream_t st)
{
    SGNN_LAUNCH(ctx, st, "ff_zero_kernel", SGNN_TAG, ff_zero_kernel, dim3(flat_blocks(rows * cols)), dim3(256), 0, st, m, rows, cols);
    return SGNN_OK;
}
