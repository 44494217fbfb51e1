// Entry points of the feed-forward operators: argument validation, scratch, and the composition of their kernels.
#include "ff.h"

namespace {

bool type_ok(const sgnn_mat *m) { return m->dtype == SGNN_F32 || m->dtype == SGNN_BF16; }
// a plain matrix of either storage type; without rows it needs no memory
bool plain(const sgnn_mat *m, int64_t rows, int64_t cols)
{
    return m && (m->ptr || rows == 0) && type_ok(m) && !m->row_index && m->rows == rows && m->cols == cols && (m->ld >= cols || rows <= 1);
}
bool plain_or_none(const sgnn_mat *m, int64_t rows, int64_t cols) { return !m || plain(m, rows, cols); }
ff_mat view(const sgnn_mat *m) { return m ? ff_mat{m->ptr, m->ld, m->dtype == SGNN_BF16} : ff_mat{nullptr, 0, 0}; }
bool is16(const sgnn_mat *m) { return m && m->dtype == SGNN_BF16; }
bool same(const sgnn_mat *a, const sgnn_mat *b) { return a && b && a->ptr && a->ptr == b->ptr; }
// one matrix as an input and the output that replaces it: laid out alike, or not the same at all
bool other_layout(const sgnn_mat *a, const sgnn_mat *b) { return same(a, b) && (a->ld != b->ld || a->dtype != b->dtype); }

constexpr int64_t FF_MAX_WIDTH = 1 << 24;

int act_ok(sgnn_ctx *ctx, const char *name, int act, int flags)
{
    if (act < SGNN_ACT_NONE || act > SGNN_ACT_SILU) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: unknown activation %d", name, act);
    if (flags & ~SGNN_BF16_MFMA) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: SGNN_BF16_MFMA is the only flag", name);
    return SGNN_OK;
}

int bind(sgnn_ctx *ctx)
{
    SGNN_HIP(ctx, hipSetDevice(ctx->device));
    return SGNN_OK;
}

int no_scratch(sgnn_ctx *ctx, const char *name) { return sgnn_fail(ctx, SGNN_ERR_CAPACITY, "%s: scratch too small: call sgnn_ctx_reserve_ffn", name); }

// m as an operand of the tile kernel: as it lies, or packed into scratch
int operand(sgnn_ctx *ctx, const char *name, const sgnn_mat *m, ws_alloc *ws, hipStream_t st, const u16 **p, int64_t *ld)
{
    if (m->dtype == SGNN_BF16 && ff_chunked(m->ptr, m->cols, m->ld)) {
        *p = static_cast<const u16 *>(m->ptr);
        *ld = m->ld;
        return SGNN_OK;
    }
    *ld = ff_pad8(m->cols);
    u16 *to = ws->get<u16>((size_t)m->rows * *ld);
    if (!ws->ok) return no_scratch(ctx, name);
    *p = to;
    return sgnn_launch_ff_pack(ctx, view(m), m->rows, m->cols, to, *ld, st);
}

const float *f32(const sgnn_mat *m) { return static_cast<const float *>(m->ptr); }
float *f32_out(const sgnn_mat *m) { return static_cast<float *>(m->ptr); }

// zeros for the gradients of weights and biases of a batch without rows
int no_rows(sgnn_ctx *ctx, int n, sgnn_mat *const *dW, float *const *db, int64_t cols, hipStream_t st)
{
    for (int q = 0; q < n; ++q) {
        if (dW[q]) {
            const int rc = sgnn_launch_ff_zero(ctx, view(dW[q]), dW[q]->rows, cols, st);
            if (rc) return rc;
        }
        if (db[q]) {
            const int rc = sgnn_launch_ff_zero(ctx, ff_mat{db[q], cols, 0}, 1, cols, st);
            if (rc) return rc;
        }
    }
    return SGNN_OK;
}

// Forward of either operator; n = 1: Y = act(X W + b) + R, n = 2: Y = act(X W0 + b0) * (X W1 + b1); Z: kept or null
int forward(sgnn_ctx *ctx, const char *name, int n, const sgnn_mat *X, const sgnn_mat *const *W, const float *const *b, int act, int flags, const sgnn_mat *R,
            sgnn_mat *Y, sgnn_mat *const *Z, sgnn_stream stream)
{
    int rc = act_ok(ctx, name, act, flags);
    if (rc) return rc;
    if (!X || !W[0] || X->rows < 0 || X->cols < 1 || W[0]->cols < 1 || X->cols > FF_MAX_WIDTH || W[0]->cols > FF_MAX_WIDTH)
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: bad argument", name);
    const int64_t M = X->rows, K = X->cols, N = W[0]->cols;
    bool ok = plain(X, M, K) && plain(Y, M, N) && plain_or_none(R, M, N);
    bool any16 = is16(X) || is16(Y) || is16(R);
    for (int q = 0; q < n; ++q) {
        ok = ok && plain(W[q], K, N) && plain_or_none(Z[q], M, N);
        any16 = any16 || is16(W[q]) || is16(Z[q]);
    }
    if (!ok) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: null pointer, shape mismatch or leading dimension too small", name);
    if (any16 && !(flags & SGNN_BF16_MFMA)) return sgnn_fail(ctx, SGNN_ERR_UNSUPPORTED, "%s: bfloat16 storage goes with SGNN_BF16_MFMA only", name);
    if (same(X, Y) || same(X, Z[0]) || same(Y, Z[0]) || same(R, Z[0]) || (n == 2 && (same(X, Z[1]) || same(Y, Z[1]) || same(Z[0], Z[1]))) ||
        other_layout(R, Y))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: an output is the same matrix as another argument", name);
    if (M == 0) return SGNN_OK;
    rc = bind(ctx);
    if (rc) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    ws_alloc ws(ctx);
    const bool b16 = (flags & SGNN_BF16_MFMA) != 0;
    ff_epilogue e = {};
    for (int q = 0; q < n; ++q) {
        e.bias[q] = b[q];
        e.Z[q] = view(Z[q]);
    }
    e.act = act;
    e.R = view(R);
    e.Y = view(Y);
    if (M <= sgnn_ff_rows_max(N, K)) {
        const ff_mat x = view(X), wv[2] = {view(W[0]), view(W[n - 1])};
        rc = sgnn_launch_ff_rows(ctx, M, N, K, 1, n, true, b16, &x, wv, e, &ws, st);
        if (rc != SGNN_ERR_UNSUPPORTED) return rc;
    }
    if (b16) {
        const u16 *a, *w[2];
        int64_t lda, ldw[2];
        rc = operand(ctx, name, X, &ws, st, &a, &lda);
        if (rc) return rc;
        for (int q = 0; q < n; ++q) {
            rc = operand(ctx, name, W[q], &ws, st, &w[q], &ldw[q]);
            if (rc) return rc;
        }
        return n == 1 ? sgnn_launch_ff_linear(ctx, M, N, K, a, lda, w[0], ldw[0], e, st) : sgnn_launch_ff_glu(ctx, M, N, K, a, lda, w[0], ldw[0], w[1], ldw[1], e, st);
    }
    // fp32: the library's split products, then the activation
    ff_mat z[2];
    for (int q = 0; q < n; ++q) {
        if (Z[q]) z[q] = view(Z[q]);
        else if (q == 1) z[q] = view(Y);          // read and written by the same thread
        else {
            float *p = ws.get<float>((size_t)M * ff_pad8(N));
            if (!ws.ok) return no_scratch(ctx, name);
            z[q] = ff_mat{p, ff_pad8(N), 0};
        }
        rc = sgnn_launch_gemm(ctx, 0, 0, M, N, K, f32(X), X->ld, nullptr, f32(W[q]), W[q]->ld, b[q], 0, static_cast<float *>(const_cast<void *>(z[q].p)), z[q].ld,
                              nullptr, 0, nullptr, &ws, st);
        if (rc) return rc;
    }
    return sgnn_launch_ff_apply(ctx, M, N, act, z[0], n == 2 ? &z[1] : nullptr, view(R), view(Y), st);
}

// Backward of either: D = the gradients of the pre-activations, then the products
int backward(sgnn_ctx *ctx, const char *name, int n, const sgnn_mat *X, const sgnn_mat *const *W, const sgnn_mat *const *Z, int act, int flags, const sgnn_mat *dY,
             sgnn_mat *dX, sgnn_mat *const *dW, float *const *db, sgnn_stream stream)
{
    int rc = act_ok(ctx, name, act, flags);
    if (rc) return rc;
    if (!X || !W[0] || !dY || X->rows < 0 || X->cols < 1 || W[0]->cols < 1 || X->cols > FF_MAX_WIDTH || W[0]->cols > FF_MAX_WIDTH)
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: bad argument", name);
    const int64_t M = X->rows, K = X->cols, N = W[0]->cols;
    const bool b16 = (flags & SGNN_BF16_MFMA) != 0, need_z = n == 2 || act != SGNN_ACT_NONE;
    bool ok = plain(X, M, K) && plain(dY, M, N) && plain_or_none(dX, M, K);
    bool any16 = is16(X) || is16(dY) || is16(dX);
    for (int q = 0; q < n; ++q) {
        ok = ok && plain(W[q], K, N) && (need_z ? plain(Z[q], M, N) : plain_or_none(Z[q], M, N)) && (!dW[q] || (plain(dW[q], K, N) && dW[q]->ptr));
        any16 = any16 || is16(W[q]) || is16(Z[q]) || is16(dW[q]);
    }
    if (!ok) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: null pointer, shape mismatch or leading dimension too small", name);
    if (any16 && !b16) return sgnn_fail(ctx, SGNN_ERR_UNSUPPORTED, "%s: bfloat16 storage goes with SGNN_BF16_MFMA only", name);
    if (same(dX, X) || same(dX, dY) || same(dX, Z[0]) || (n == 2 && (same(dX, Z[1]) || same(dW[0], dW[1]))))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: an output is the same matrix as another argument", name);
    const bool any_dw = dW[0] || (n == 2 && dW[1]), any_db = db[0] || (n == 2 && db[1]);
    if (!dX && !any_dw && !any_db) return SGNN_OK;
    rc = bind(ctx);
    if (rc) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (M == 0) return no_rows(ctx, n, dW, db, N, st);
    ws_alloc ws(ctx);
    // [D0 | D1] in one matrix, each padded with zeros to whole 16-byte chunks
    const int64_t np = ff_pad8(N), ldd = n * np;
    void *D = b16 ? static_cast<void *>(ws.get<u16>((size_t)M * ldd)) : static_cast<void *>(ws.get<float>((size_t)M * ldd));
    if (!ws.ok) return no_scratch(ctx, name);
    const ff_mat d0 = {D, ldd, b16}, d1 = {b16 ? static_cast<void *>(static_cast<u16 *>(D) + np) : static_cast<void *>(static_cast<float *>(D) + np), ldd, b16};
    const ff_mat z0 = need_z ? view(Z[0]) : view(dY), z1 = n == 2 ? view(Z[1]) : ff_mat{};
    rc = sgnn_launch_ff_act_bwd(ctx, M, N, np, act, view(dY), z0, n == 2 ? &z1 : nullptr, d0, n == 2 ? &d1 : nullptr, db, &ws, st);
    if (rc) return rc;
    // the gradient of a few rows; dX, if it is still wanted, by the tile kernels
    auto few_rows = [&]() -> int {
        if (!dX || M > sgnn_ff_rows_max(K, n * N)) return SGNN_ERR_UNSUPPORTED;
        ff_epilogue e = {};
        e.Y = view(dX);
        const ff_mat x[2] = {d0, n == 2 ? d1 : d0}, wv[2] = {view(W[0]), view(W[n - 1])};
        return sgnn_launch_ff_rows(ctx, M, K, N, n, 1, false, b16, x, wv, e, &ws, st);
    };
    rc = few_rows();
    if (rc != SGNN_OK && rc != SGNN_ERR_UNSUPPORTED) return rc;
    if (rc == SGNN_OK) dX = nullptr;
    rc = SGNN_OK;
    if (b16) {
        const u16 *dp[2] = {static_cast<const u16 *>(d0.p), static_cast<const u16 *>(d1.p)};
        if (any_dw) {
            const size_t off = ws.off;
            const u16 *a;
            int64_t lda;
            rc = operand(ctx, name, X, &ws, st, &a, &lda);
            if (rc) return rc;
            // both results of one launch, or the one that is wanted
            const u16 *bp[2];
            ff_mat c[2];
            int mats = 0;
            for (int q = 0; q < n; ++q)
                if (dW[q]) { bp[mats] = dp[q]; c[mats++] = view(dW[q]); }
            rc = sgnn_launch_ff_tn(ctx, K, N, M, mats, a, lda, bp, ldd, c, &ws, st);
            if (rc) return rc;
            ws.off = off;
        }
        if (dX) {
            const u16 *w[2];
            int64_t ldw[2];
            for (int q = 0; q < n; ++q) {
                rc = operand(ctx, name, W[q], &ws, st, &w[q], &ldw[q]);
                if (rc) return rc;
            }
            if (n == 2 && ldw[0] != ldw[1]) {       // one leading dimension for both
                for (int q = 0; q < 2; ++q) {
                    u16 *to = ws.get<u16>((size_t)K * np);
                    if (!ws.ok) return no_scratch(ctx, name);
                    rc = sgnn_launch_ff_pack(ctx, view(W[q]), K, N, to, np, st);
                    if (rc) return rc;
                    w[q] = to;
                    ldw[q] = np;
                }
            }
            rc = sgnn_launch_ff_nt(ctx, M, K, N, n, dp, ldd, w, ldw[0], view(dX), st);
        }
        return rc;
    }
    for (int q = 0; q < n; ++q)
        if (dW[q]) {
            rc = sgnn_launch_gemm(ctx, 1, 0, K, N, M, f32(X), X->ld, nullptr, static_cast<const float *>(q ? d1.p : d0.p), ldd, nullptr, 0, f32_out(dW[q]), dW[q]->ld,
                                  nullptr, 0, nullptr, &ws, st);
            if (rc) return rc;
        }
    if (!dX) return SGNN_OK;
    const float *w = f32(W[0]);
    int64_t ldw = W[0]->ld, kk = N;
    if (n == 2) {
        // [W0 | W1], so that the sum over both is one product
        float *to = ws.get<float>((size_t)K * ldd);
        if (!ws.ok) return no_scratch(ctx, name);
        for (int q = 0; q < 2; ++q) {
            rc = sgnn_launch_ff_copy32(ctx, f32(W[q]), W[q]->ld, K, N, np, to + q * np, ldd, st);
            if (rc) return rc;
        }
        w = to;
        ldw = kk = ldd;
    }
    return sgnn_launch_gemm(ctx, 0, 1, M, K, kk, static_cast<const float *>(D), ldd, nullptr, w, ldw, nullptr, 0, f32_out(dX), dX->ld, nullptr, 0, nullptr, &ws, st);
}

} // namespace

extern "C" {

int sgnn_ctx_reserve_ffn(sgnn_ctx *ctx, uint64_t rows, uint32_t d_in, uint32_t d_out)
{
    if (!ctx) return SGNN_ERR_INVALID_ARG;
    if (d_in > FF_MAX_WIDTH || d_out > FF_MAX_WIDTH || rows >= (1ull << 40)) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "sgnn_ctx_reserve_ffn: bad argument");
    int rc = bind(ctx);
    if (rc) return rc;
    const uint64_t di = ff_pad8(d_in), dn = ff_pad8(d_out);
    // fp32 split products: at most 256 ranges of the reduction, and 2304 tiles of 256 x 128 over all ranges
    const uint64_t split = std::min<uint64_t>(2304ull * 256 * 128 * 4, d_in >= 4096 || d_out >= 4096 ? ~0ull : 257 * 4 * di * dn) + 257 * 4 * std::max(di, dn);
    size_t need = rows * (2 * dn * 4 + di * 2) + 2 * di * dn * 4 * 2 + split + sgnn_ff_tn_ws_bytes(rows, di, dn) + sgnn_ff_sums_ws_bytes(dn) + sgnn_ff_rows_ws_bytes() + 16 * 256;
    need = std::max(need, sgnn_block_norm_ws_bytes(std::max(d_in, d_out)));
    if (need > ctx->ws_bytes) {
        SGNN_HIP(ctx, hipDeviceSynchronize());
        if (ctx->ws) SGNN_HIP(ctx, hipFree(ctx->ws));
        ctx->ws = nullptr;
        ctx->ws_bytes = 0;
        SGNN_HIP(ctx, hipMalloc(&ctx->ws, need));
        ctx->ws_bytes = need;
    }
    return SGNN_OK;
}

int sgnn_linear_fwd(sgnn_ctx *ctx, const sgnn_mat *X, const sgnn_mat *W, const float *bias, int act, int flags, const sgnn_mat *R, sgnn_mat *Y, sgnn_mat *Z,
                    sgnn_stream stream)
{
    if (!ctx) return SGNN_ERR_INVALID_ARG;
    const sgnn_mat *w[2] = {W, nullptr};
    const float *b[2] = {bias, nullptr};
    sgnn_mat *z[2] = {Z, nullptr};
    return forward(ctx, "sgnn_linear_fwd", 1, X, w, b, act, flags, R, Y, z, stream);
}

int sgnn_linear_bwd(sgnn_ctx *ctx, const sgnn_mat *X, const sgnn_mat *W, const sgnn_mat *Z, int act, int flags, const sgnn_mat *dY, sgnn_mat *dX, sgnn_mat *dW,
                    float *dbias, sgnn_stream stream)
{
    if (!ctx) return SGNN_ERR_INVALID_ARG;
    const sgnn_mat *w[2] = {W, nullptr}, *z[2] = {Z, nullptr};
    sgnn_mat *dw[2] = {dW, nullptr};
    float *db[2] = {dbias, nullptr};
    return backward(ctx, "sgnn_linear_bwd", 1, X, w, z, act, flags, dY, dX, dw, db, stream);
}

int sgnn_glu_fwd(sgnn_ctx *ctx, const sgnn_mat *X, const sgnn_mat *Wg, const sgnn_mat *Wu, const float *bg, const float *bu, int act, int flags, sgnn_mat *H,
                 sgnn_mat *G, sgnn_mat *U, sgnn_stream stream)
{
    if (!ctx) return SGNN_ERR_INVALID_ARG;
    const sgnn_mat *w[2] = {Wg, Wu};
    const float *b[2] = {bg, bu};
    sgnn_mat *z[2] = {G, U};
    return forward(ctx, "sgnn_glu_fwd", 2, X, w, b, act, flags, nullptr, H, z, stream);
}

int sgnn_glu_bwd(sgnn_ctx *ctx, const sgnn_mat *X, const sgnn_mat *Wg, const sgnn_mat *Wu, const sgnn_mat *G, const sgnn_mat *U, int act, int flags,
                 const sgnn_mat *dH, sgnn_mat *dX, sgnn_mat *dWg, sgnn_mat *dWu, float *dbg, float *dbu, sgnn_stream stream)
{
    if (!ctx) return SGNN_ERR_INVALID_ARG;
    const sgnn_mat *w[2] = {Wg, Wu}, *z[2] = {G, U};
    sgnn_mat *dw[2] = {dWg, dWu};
    float *db[2] = {dbg, dbu};
    return backward(ctx, "sgnn_glu_bwd", 2, X, w, z, act, flags, dH, dX, dw, db, stream);
}

static int norm_args(sgnn_ctx *ctx, const char *name, const sgnn_block_norm *p, int64_t rows, int64_t d, const sgnn_mat *Z, ff_norm *a)
{
    if (!p || d < 1 || rows < 0 || !(p->eps >= 0.f)) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: bad argument", name);
    if (p->gate && !plain(p->gate, rows, 1) && !plain(p->gate, rows, d))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: the gate has one column, or as many as the matrices", name);
    if (!Z && (p->gate || p->gamma_post || p->col_scale || p->post))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: gate, scale and norm of a block without its output Z", name);
    if (!p->post && p->gamma_post) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: gamma_post without the norm it scales", name);
    *a = ff_norm{};
    a->rows = rows;
    a->d = (int)std::min<int64_t>(d, 0x7fffffff);
    a->z = view(Z);
    a->gate = view(p->gate);
    a->gate_cols = p->gate ? (int)p->gate->cols : 0;
    a->gamma_post = p->gamma_post;
    a->scale = p->col_scale;
    a->gamma_pre = p->gamma_pre;
    a->alpha = p->res_scale;
    a->eps = p->eps;
    a->post = p->post ? 1 : 0;
    return SGNN_OK;
}

int sgnn_block_norm_fwd(sgnn_ctx *ctx, const sgnn_mat *X, const sgnn_mat *Z, const sgnn_block_norm *p, sgnn_mat *Y, sgnn_mat *N, float *inv_rms_post,
                        float *inv_rms_pre, sgnn_stream stream)
{
    if (!ctx) return SGNN_ERR_INVALID_ARG;
    if (!X || (!Y && !N)) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "sgnn_block_norm_fwd: X and one of Y and N are needed");
    const int64_t rows = X->rows, d = X->cols;
    if (!plain(X, rows, d) || !plain_or_none(Z, rows, d) || !plain_or_none(Y, rows, d) || !plain_or_none(N, rows, d))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "sgnn_block_norm_fwd: null pointer, shape mismatch or leading dimension too small");
    ff_norm a;
    int rc = norm_args(ctx, "sgnn_block_norm_fwd", p, rows, d, Z, &a);
    if (rc) return rc;
    if ((inv_rms_post && !(p->post && Z)) || (inv_rms_pre && !N) || same(Y, N) || other_layout(X, Y) || other_layout(X, N) || other_layout(Z, Y) || other_layout(Z, N))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "sgnn_block_norm_fwd: the inverse root of a norm that is not taken, or one matrix for two arguments");
    if (rows == 0) return SGNN_OK;
    rc = bind(ctx);
    if (rc) return rc;
    a.x = view(X); a.y = view(Y); a.n = view(N);
    a.ir_post = inv_rms_post; a.ir_pre = inv_rms_pre;
    return sgnn_launch_block_norm_fwd(ctx, a, static_cast<hipStream_t>(stream));
}

int sgnn_block_norm_bwd(sgnn_ctx *ctx, const sgnn_mat *Z, const sgnn_mat *Y, const sgnn_block_norm *p, const float *inv_rms_post, const float *inv_rms_pre,
                        const sgnn_mat *dY, const sgnn_mat *dN, sgnn_mat *dX, sgnn_mat *dZ, sgnn_mat *dgate, float *dgamma_post, float *dscale, float *dgamma_pre,
                        sgnn_stream stream)
{
    if (!ctx) return SGNN_ERR_INVALID_ARG;
    const sgnn_mat *in = dY ? dY : dN;
    if (!in) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "sgnn_block_norm_bwd: dY or dN is needed");
    const int64_t rows = in->rows, d = in->cols;
    if (!plain(in, rows, d) || !plain_or_none(dY, rows, d) || !plain_or_none(dN, rows, d) || !plain_or_none(Z, rows, d) || !plain_or_none(Y, rows, d) ||
        !plain_or_none(dX, rows, d) || !plain_or_none(dZ, rows, d))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "sgnn_block_norm_bwd: null pointer, shape mismatch or leading dimension too small");
    ff_norm a;
    int rc = norm_args(ctx, "sgnn_block_norm_bwd", p, rows, d, Z, &a);
    if (rc) return rc;
    if (rows > 0 && ((dN && (!Y || !inv_rms_pre)) || (Z && p->post && !inv_rms_post)))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "sgnn_block_norm_bwd: a norm's input and inverse root are needed for its backward pass");
    if ((!Z && (dZ || dscale)) || (dgate && (!p->gate || !plain(dgate, rows, p->gate->cols))) || (dgamma_post && !p->post) || (dgamma_pre && !dN))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "sgnn_block_norm_bwd: the gradient of something the block does not have");
    bool twice = same(dX, dZ) || same(dgate, dX) || same(dgate, dZ);
    for (const sgnn_mat *o : {static_cast<const sgnn_mat *>(dX), static_cast<const sgnn_mat *>(dZ)})
        for (const sgnn_mat *i : {dY, dN, Z, Y}) twice = twice || other_layout(i, o);
    if (twice) return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "sgnn_block_norm_bwd: one matrix for two arguments");
    rc = bind(ctx);
    if (rc) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows == 0) {
        sgnn_mat *none[1] = {nullptr};
        for (float *v : {dgamma_post, dscale, dgamma_pre}) {
            float *const db[1] = {v};
            rc = no_rows(ctx, 1, none, db, d, st);
            if (rc) return rc;
        }
        return SGNN_OK;
    }
    a.dy = view(dY); a.dn = view(dN); a.dx = view(dX); a.dz = view(dZ); a.dgate = view(dgate);
    if (dN) a.y = view(Y);
    a.in_ir_post = inv_rms_post; a.in_ir_pre = inv_rms_pre;
    a.dgamma_post = dgamma_post; a.dscale = dscale; a.dgamma_pre = dgamma_pre;
    ws_alloc ws(ctx);
    return sgnn_launch_block_norm_bwd(ctx, a, &ws, st);
}

} // extern "C"
