// What the kernels of the feed-forward operators (ff_*.hip, block_norm.hip) share.
#pragma once

#include <algorithm>
#include <type_traits>

#include "gemm_stream.h"

// 16 bytes of either storage type at any alignment of their elements (gfx950 global loads and stores take any)
typedef u32x4 u32x4_any2 __attribute__((aligned(2)));

// a matrix as the kernels see it
struct ff_mat { const void *p; int64_t ld; int b16; };

__device__ __forceinline__ float ff_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float ff_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

// an operand's eight values from LDS; __restrict__ for the reason given at read_tr
__device__ __forceinline__ u32x4 read_row(const unsigned char *__restrict__ p) { return *reinterpret_cast<const u32x4 *>(p); }

// storage of a matrix: known when the kernel is compiled, or a field of its arguments
enum { FF_T32 = 0, FF_T16 = 1, FF_TANY = 2 };

// v[0 .. N) = row elements at (row, col), of which `left` exist (the others are 0)
template <int T, int N> __device__ __forceinline__ void ff_load(float (&v)[N], const ff_mat &m, int64_t row, int64_t col, int left)
{
    const bool b16 = T == FF_TANY ? m.b16 != 0 : T == FF_T16;
    if (b16) {
        const u16 *p = static_cast<const u16 *>(m.p) + row * m.ld + col;
        if (N == 8 && left >= 8) {
            const u32x4 w = *reinterpret_cast<const u32x4_any2 *>(p);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) { v[2 * i] = ff_lo(w[i % 4]); v[2 * i + 1] = ff_hi(w[i % 4]); }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = i < left ? __builtin_bit_cast(float, (uint32_t)p[i] << 16) : 0.f;
        }
    } else {
        const float *p = static_cast<const float *>(m.p) + row * m.ld + col;
        if (left >= N) {
#pragma unroll
            for (int q = 0; q < N / 4; ++q) {
                const f32x4 w = *reinterpret_cast<const f32x4_any *>(p + 4 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[4 * q + i] = w[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = i < left ? p[i] : 0.f;
        }
    }
}

// the same the other way; bfloat16 is rounded to nearest even
template <int T, int N> __device__ __forceinline__ void ff_store(const float (&v)[N], const ff_mat &m, int64_t row, int64_t col, int left)
{
    const bool b16 = T == FF_TANY ? m.b16 != 0 : T == FF_T16;
    if (b16) {
        u16 *p = static_cast<u16 *>(const_cast<void *>(m.p)) + row * m.ld + col;
        if (N == 8 && left >= 8) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < N / 2; ++i) w[i % 4] = pack_bf16(v[2 * i], v[2 * i + 1]);
            *reinterpret_cast<u32x4_any2 *>(p) = w;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < left) p[i] = __builtin_bit_cast(u16, (__bf16)v[i]);
        }
    } else {
        float *p = static_cast<float *>(const_cast<void *>(m.p)) + row * m.ld + col;
        if (left >= N) {
#pragma unroll
            for (int q = 0; q < N / 4; ++q) *reinterpret_cast<f32x4_any *>(p + 4 * q) = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < left) p[i] = v[i];
        }
    }
}

static inline int64_t ff_pad8(int64_t n) { return (n + 7) & ~int64_t(7); }
// the tile kernel takes the matrix as it lies: 16-byte chunks along a row are whole ones, and a tile's offsets fit 32 bits
static inline bool ff_chunked(const void *p, int64_t cols, int64_t ld)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && cols % 8 == 0 && ld % 8 == 0 && ld <= (1 << 22);
}

// The context's counts of arrivals, zero between calls
static inline uint32_t *sgnn_ff_arrived(sgnn_ctx *ctx) { return reinterpret_cast<uint32_t *>(ctx->persist + SGNN_PERSIST_FFN_OFF); }
static inline int sgnn_ff_open(sgnn_ctx *ctx, hipStream_t st) { return sgnn_zero_open(ctx, SGNN_ZERO_FFN, ctx->persist + SGNN_PERSIST_FFN_OFF, SGNN_PERSIST_FFN_BYTES, st); }
static inline int sgnn_ff_close(sgnn_ctx *ctx, int rc, hipStream_t st) { return sgnn_zero_close(ctx, rc, SGNN_ZERO_FFN, ctx->persist + SGNN_PERSIST_FFN_OFF, SGNN_PERSIST_FFN_BYTES, st); }

// ---- ff_gemm.hip: products of any size ----------------------------------------------------------
struct ff_epilogue {
    int act;                          // SGNN_ACT_*
    const float *bias[2];             // of each projection, or null
    ff_mat R, Y, Z[2];                // residual, result, pre-activations kept (p may be null but for Y)
};
// an operand, chunked (ff_chunked): bfloat16 (pl = 1), or fp16 parts (pl = 2: fp32), eight first ones and eight second ones in turn.  ex_rows, ex: the scales of the
// rows of A, if they have their own, and of everything else (of both operands together)
struct ff_op { const u16 *p; int64_t ld; };        // ld in elements of 16 bits
// Y = act(A B + bias) + R, with mats = 2 Y = act(A B0 + bias0) * (A B1 + bias1); A [M x K], B [K x N]; the epilogue's matrices as they come
int sgnn_launch_ff_nn(sgnn_ctx *ctx, int pl, int64_t M, int64_t N, int64_t K, int mats, const ff_op &A, const ff_op *B, const int32_t *ex_rows, const int32_t *ex,
                      const ff_epilogue &e, ws_alloc *ws, hipStream_t st);
// Y = sum over s < segs of A[s] B[s]^T; A[s] [M x K], B[s] [N x K], laid out alike
int sgnn_launch_ff_nt(sgnn_ctx *ctx, int pl, int64_t M, int64_t N, int64_t K, int segs, const ff_op *A, const ff_op *B, const int32_t *ex_rows, const int32_t *ex,
                      const ff_mat &Y, ws_alloc *ws, hipStream_t st);
// D[s], the gradients of the pre-activations Z (side by side in D [M x mats N], or D null), and dX [M x K] = sum over s of D[s] W[s]^T; or SGNN_ERR_UNSUPPORTED
int sgnn_launch_ff_dx(sgnn_ctx *ctx, int64_t M, int64_t N, int64_t K, int mats, int act, const ff_mat &dY, const ff_mat *Z, const ff_op *W, const ff_mat &D, const ff_mat &dX,
                      hipStream_t st);
// C[s] = A^T B[s] for s < mats; A [K x M], B[s] [K x N], laid out alike
int sgnn_launch_ff_tn(sgnn_ctx *ctx, int pl, int64_t M, int64_t N, int64_t K, int mats, const ff_op &A, const ff_op *B, const int32_t *ex_rows, const int32_t *ex,
                      const ff_mat *C, ws_alloc *ws, hipStream_t st);
size_t sgnn_ff_gemm_ws_bytes(uint64_t d_in, uint64_t d_out);

// ---- ff_rows.hip: the same for a few rows, matrices as they come ----------------------------------
// nn: weights [K x N] (two: gated); else nt over segs segments.  SGNN_ERR_UNSUPPORTED (nothing launched) for projections stored differently
int sgnn_launch_ff_rows(sgnn_ctx *ctx, int64_t M, int64_t N, int64_t K, int segs, int mats, bool nn, bool b16, const ff_mat *X, const ff_mat *W, const ff_epilogue &e,
                        ws_alloc *ws, hipStream_t st);
bool sgnn_ff_rows_take(bool b16, int64_t M, int64_t N, int64_t K, int mats);
size_t sgnn_ff_rows_ws_bytes();

// ---- ff_elem.hip --------------------------------------------------------------------------------
// dst [rows x ff_pad8(cols)] = src in bfloat16, zeros behind the last column
int sgnn_launch_ff_pack(sgnn_ctx *ctx, const ff_mat &src, int64_t rows, int64_t cols, u16 *dst, int64_t ldd, hipStream_t st);
// dst = src in dst's storage
int sgnn_launch_ff_convert(sgnn_ctx *ctx, const ff_mat &src, int64_t rows, int64_t cols, const ff_mat &dst, hipStream_t st);
// fp32 operands as fp16 parts [rows x 2 ff_pad8(cols)], zeros behind the last column (ff_gemm.hip says how and why).
struct ff_scan { const float *p; int64_t rows, cols, ld; };
// The rows of one matrix, each scaled by a power of two of its own: 2^ex[row] takes the row's largest finite magnitude to [2^14, 2^15); FF_EX_ZERO
// for a row without one.  to null: the exponents only.  With `other`, the exponents of another matrix' rows, every workgroup (sgnn_ff_row_groups of them)
// leaves the largest FF_EX_KEY - ex[row] - other[row] of its rows in a word of key.  The same launch finds the largest finite magnitudes of up to two weight
// matrices: a word of largest, its bits, for every workgroup (sgnn_ff_scan_groups for each matrix).
struct ff_row_parts { ff_scan m; u16 *to; int64_t ld; int32_t *ex; const int32_t *other; uint32_t *key; };
constexpr int FF_EX_ZERO = 2000, FF_EX_KEY = 8192, FF_ROW_WORDS = 4096, FF_SCAN_WORDS = 512;
unsigned sgnn_ff_row_groups(int64_t rows, int64_t cols);
unsigned sgnn_ff_scan_groups(int n, const ff_scan *w);
int sgnn_launch_ff_row_parts(sgnn_ctx *ctx, const ff_row_parts &r, int n, const ff_scan *w, uint32_t *largest, hipStream_t st);
// Up to three matrices with the scale known from such words: rows == null, one scale for the matrix; else FF_EX_KEY - largest word - rows[row] for
// each row.  *ex: the scale of the matrix, or FF_EX_KEY - largest word
struct ff_parts { ff_scan m; const uint32_t *word; int words; const int32_t *rows; int32_t *ex; u16 *to; int64_t ld; };
int sgnn_launch_ff_parts(sgnn_ctx *ctx, int n, const ff_parts *m, hipStream_t st);
// (D0 without memory: the column sums only)
// D0 = dY * act'(Z0), or with Z1 D0 = dY * Z1 * act'(Z0) and D1 = dY * act(Z0); zeros in the columns from cols to pcols; column sums (before
// the rounding) to db[0], db[1] where they are wanted
int sgnn_launch_ff_act_bwd(sgnn_ctx *ctx, int64_t rows, int64_t cols, int64_t pcols, int act, const ff_mat &dY, const ff_mat &Z0, const ff_mat *Z1,
                           const ff_mat &D0, const ff_mat *D1, float *const *db, ws_alloc *ws, hipStream_t st);
// The same of fp32 matrices straight into the parts of [D0 | D1] (p.to, p.ld, and p.ex, p.other, p.key as above, a word of key for each of the groups)
unsigned sgnn_ff_act_bwd_parts_groups(int64_t rows, int64_t pcols);
int sgnn_launch_ff_act_bwd_parts(sgnn_ctx *ctx, int64_t rows, int64_t cols, int64_t pcols, int act, const ff_mat &dY, const ff_mat &Z0, const ff_mat *Z1,
                                 const ff_row_parts &p, float *const *db, ws_alloc *ws, hipStream_t st);
// zeros; rows of ld elements, cols of them written
int sgnn_launch_ff_zero(sgnn_ctx *ctx, const ff_mat &m, int64_t rows, int64_t cols, hipStream_t st);
size_t sgnn_ff_sums_ws_bytes(uint64_t cols);

// ---- block_norm.hip -----------------------------------------------------------------------------
struct ff_norm {
    int64_t rows;
    int d;
    ff_mat x, z, gate, y, n;          // p null where there is none
    int gate_cols;                    // 1 or d
    const float *gamma_post, *scale, *gamma_pre;
    float alpha, eps;
    int post;
    float *ir_post, *ir_pre;
    // backward
    ff_mat dy, dn, dx, dz, dgate;
    const float *in_ir_post, *in_ir_pre;
    float *dgamma_post, *dscale, *dgamma_pre;
};
int sgnn_launch_block_norm_fwd(sgnn_ctx *ctx, const ff_norm &a, hipStream_t st);
int sgnn_launch_block_norm_bwd(sgnn_ctx *ctx, const ff_norm &a, ws_alloc *ws, hipStream_t st);
size_t sgnn_block_norm_ws_bytes(uint64_t d);
