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

// an output that is the same matrix as an input, or as another output
bool clash(std::initializer_list<const sgnn_mat *> outs, std::initializer_list<const sgnn_mat *> ins)
{
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        for (const sgnn_mat *i : ins)
            if (same(*o, i)) return true;
        for (auto p = o + 1; p != outs.end(); ++p)
            if (same(*o, *p)) return true;
    }
    return false;
}

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

// m as a bfloat16 operand of the tile kernels: as it lies, or packed into scratch (always with `pack`)
int operand(sgnn_ctx *ctx, const char *name, const sgnn_mat *m, bool pack, ws_alloc *ws, hipStream_t st, ff_op *op)
{
    if (!pack && m->dtype == SGNN_BF16 && ff_chunked(m->ptr, m->cols, m->ld)) {
        *op = ff_op{static_cast<const u16 *>(m->ptr), m->ld};
        return SGNN_OK;
    }
    const int64_t ld = ff_pad8(m->cols);
    u16 *to = ws->get<u16>((size_t)m->rows * ld);
    if (!ws->ok) return no_scratch(ctx, name);
    *op = ff_op{to, ld};
    return sgnn_launch_ff_pack(ctx, view(m), m->rows, m->cols, to, ld, st);
}

ff_scan scan(const sgnn_mat *m) { return ff_scan{static_cast<const float *>(m->ptr), m->rows, m->cols, m->ld}; }

// scratch for the parts of an fp32 matrix
ff_op parts_op(ws_alloc *ws, int64_t rows, int64_t cols)
{
    const int64_t ld = 2 * ff_pad8(cols);
    return ff_op{ws->get<u16>((size_t)rows * ld), ld};
}

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
    if (clash({Y, Z[0], n == 2 ? Z[1] : nullptr}, {X, W[0], n == 2 ? W[1] : nullptr}) || same(R, Z[0]) || other_layout(R, Y))
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
    if (sgnn_ff_rows_take(b16, M, N, K, n)) {
        const ff_mat xv = view(X), wv[2] = {view(W[0]), view(W[n - 1])};
        rc = sgnn_launch_ff_rows(ctx, M, N, K, 1, n, true, b16, &xv, wv, e, &ws, st);
        if (rc != SGNN_ERR_UNSUPPORTED) return rc;
    }
    ff_op x, w[2];
    if (b16) {
        rc = operand(ctx, name, X, false, &ws, st, &x);
        for (int q = 0; q < n && !rc; ++q) rc = operand(ctx, name, W[q], false, &ws, st, &w[q]);
        if (rc) return rc;
        return sgnn_launch_ff_nn(ctx, 1, M, N, K, n, x, w, nullptr, nullptr, e, &ws, st);
    }
    // fp32.  A product of at most 256 tiles of 256 x 128, one a compute unit, with a short K, or onto few columns: three parts split as X is
    // read and six products (gemm_split.hip) cost less than two parts of X made first, 8 bytes a value at the rate of a copy and two launches, and three
    // products.  With Z and R, parts first against split as read: 32768 x 256 x 256 50 and 44 us, 131072 x 512 x 128 204 and 147, 8192 x 256 x 512 38
    // and 27, 15167 x 3762 x 27 194 and 90, 2500 x 1024 x 64 31 and 17; past the rule 131072 x 256 x 256 171 and 196, 32768 x 256 x 512 67 and 86, 4096 x 2048 x 256
    // 48 and 71
    if (n == 1 && K >= 4 && N >= 4 && ((K <= 512 && ((M + 255) / 256) * ((N + 127) / 128) <= 256) || N <= 128)) {
        const sgnn_split_epilogue se = {1, act, R ? static_cast<const float *>(R->ptr) : nullptr, R ? R->ld : 0, Z[0] ? static_cast<float *>(Z[0]->ptr) : nullptr, Z[0] ? Z[0]->ld : 0};
        return sgnn_launch_gemm_split(ctx, 0, 0, M, N, K, static_cast<const float *>(X->ptr), X->ld, nullptr, static_cast<const float *>(W[0]->ptr), W[0]->ld, b[0], 0,
                                      static_cast<float *>(Y->ptr), Y->ld, nullptr, 0, nullptr, &ws, st, &se);
    }
    // the rows of X scaled by themselves, the weights by their largest value (ff_gemm.hip)
    ff_scan scans[2];
    ff_parts job[2];
    x = parts_op(&ws, M, K);
    int32_t *const ex_rows = ws.get<int32_t>((size_t)M + 1), *const ex = ex_rows + M;
    uint32_t *const largest = ws.get<uint32_t>(2 * FF_SCAN_WORDS);
    for (int q = 0; q < n; ++q) {
        w[q] = parts_op(&ws, K, N);
        scans[q] = scan(W[q]);
    }
    if (!ws.ok) return no_scratch(ctx, name);
    const int words = n * (int)sgnn_ff_scan_groups(n, scans);
    for (int q = 0; q < n; ++q) job[q] = ff_parts{scans[q], largest, words, nullptr, ex, const_cast<u16 *>(w[q].p), w[q].ld};
    rc = sgnn_launch_ff_row_parts(ctx, ff_row_parts{scan(X), const_cast<u16 *>(x.p), x.ld, ex_rows, nullptr, nullptr}, n, scans, largest, st);
    if (!rc) rc = sgnn_launch_ff_parts(ctx, n, job, st);
    return rc ? rc : sgnn_launch_ff_nn(ctx, 2, M, N, K, n, x, w, ex_rows, ex, e, &ws, st);
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
    const bool two = n == 2;
    if (clash({dX, dW[0], two ? dW[1] : nullptr}, {X, dY, Z[0], W[0], two ? Z[1] : nullptr, two ? W[1] : nullptr}))
        return sgnn_fail(ctx, SGNN_ERR_INVALID_ARG, "%s: an output is the same matrix as another argument", name);
    const bool any_dw = dW[0] || (n == 2 && dW[1]), any_db = db[0] || (n == 2 && db[1]);
    if (!dX && !any_dw && !any_db) return SGNN_OK;
    rc = bind(ctx);
    if (rc) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (M == 0) return no_rows(ctx, n, dW, db, N, st);
    ws_alloc ws(ctx);
    // [D0 | D1] in one matrix, each padded with zeros to whole 16-byte chunks; without an activation dY itself, if the products can read it
    const bool is_dy = !need_z && (!b16 || (is16(dY) && ff_chunked(dY->ptr, N, dY->ld)));
    const int64_t np = is_dy ? N : ff_pad8(N), ldd = is_dy ? dY->ld : n * np;
    // (fp32: not written where the gradients become parts at once, see below)
    void *D = is_dy ? dY->ptr : (b16 ? static_cast<void *>(ws.get<u16>((size_t)M * ldd)) : static_cast<void *>(ws.get<float>((size_t)M * ldd)));
    if (!ws.ok) return no_scratch(ctx, name);
    const ff_mat d0 = {D, ldd, b16}, d1 = {b16 ? static_cast<void *>(static_cast<u16 *>(D) + np) : static_cast<void *>(static_cast<float *>(D) + np), ldd, b16};
    const ff_mat z0 = need_z ? view(Z[0]) : view(dY), z1 = n == 2 ? view(Z[1]) : ff_mat{};
    auto gradients = [&]() -> int {
        if (is_dy && !any_db) return SGNN_OK;
        return sgnn_launch_ff_act_bwd(ctx, M, N, np, act, view(dY), z0, n == 2 ? &z1 : nullptr, is_dy ? ff_mat{nullptr, 0, b16} : d0, n == 2 ? &d1 : nullptr, db, &ws, st);
    };
    const bool few = dX && sgnn_ff_rows_take(b16, M, K, n * N, 1);
    // the gradient of a few rows
    auto few_rows = [&]() -> int {
        ff_epilogue e = {};
        e.Y = view(dX);
        const ff_mat xv[2] = {d0, n == 2 ? d1 : d0}, wv[2] = {view(W[0]), view(W[n - 1])};
        return sgnn_launch_ff_rows(ctx, M, K, N, n, 1, false, b16, xv, wv, e, &ws, st);
    };
    // both weight gradients in one launch, or the one that is wanted
    auto weights = [&](int pl, const ff_op &x, const ff_op *d, const int32_t *ex_x, const int32_t *ex_d) -> int {
        ff_op b[2];
        ff_mat c[2];
        int mats = 0;
        for (int q = 0; q < n; ++q)
            if (dW[q]) { b[mats] = d[q]; c[mats++] = view(dW[q]); }
        return sgnn_launch_ff_tn(ctx, pl, K, N, M, mats, x, b, ex_x, ex_d, c, &ws, st);
    };
    ff_op x, w[2];
    if (b16) {
        // two projections laid out alike, by packing both if they are not
        const bool pack = n == 2 && (W[0]->ld != W[1]->ld || is16(W[0]) != is16(W[1]) || ff_chunked(W[0]->ptr, N, W[0]->ld) != ff_chunked(W[1]->ptr, N, W[1]->ld));
        auto weight_operands = [&]() -> int {
            for (int q = 0; q < n; ++q) {
                const int e = operand(ctx, name, W[q], pack, &ws, st, &w[q]);
                if (e) return e;
            }
            return SGNN_OK;
        };
        bool dx_done = false;
        // D and dX in one pass (ff_dx.hip), where no sums over the rows of D are asked for.  A workgroup has 128 rows: it takes many of them, or few steps each.  Both
        // operators' whole backward passes with it and without, us: gated, 256 columns of X, 704 of W, 131072 rows 348 and 438, 32768 96 and 125, 16384
        // 68 and 72, 8192 60 and 56; 8192 x 256 x 128 26.7 and 27.1; linear 131072 x 256 x 512 186 and 214, 32768 x 256 x 256 41 and 61, 8192 x 256 x 256
        // 31 and 50, 16384 x 128 x 1024 69 and 63.  A linear pass onto up to 128 columns of many rows has both products in one already (below):
        // 131072 x 256 x 128 87 and 81, 49152 x 256 x 128 47 and 53.
        if (dX && !few && !any_db && need_z && K <= 256 && (M >= 32768 || (M >= 8192 && K > 128 && N <= 512)) && !(n == 1 && N <= 128 && M >= 65536)) {
            const size_t off = ws.off;
            const ff_mat z[2] = {z0, z1};
            rc = weight_operands();
            if (!rc) rc = sgnn_launch_ff_dx(ctx, M, N, K, n, act, view(dY), z, w, any_dw ? d0 : ff_mat{nullptr, 0, 1}, view(dX), st);
            if (rc != SGNN_OK && rc != SGNN_ERR_UNSUPPORTED) return rc;
            dx_done = rc == SGNN_OK;
            ws.off = off;
        }
        if (!dx_done) rc = gradients();
        if (rc) return rc;
        if (few) {
            rc = few_rows();
            if (rc != SGNN_OK && rc != SGNN_ERR_UNSUPPORTED) return rc;
            dx_done = rc == SGNN_OK;
        }
        const ff_op d[2] = {{static_cast<const u16 *>(d0.p), ldd}, {static_cast<const u16 *>(d1.p), ldd}};
        // both products of many rows onto up to 256 columns in one pass over X and D (gemm_bwd.hip)
        if (n == 1 && dX && dW[0] && !dx_done && is16(X) && is16(dX)) {
            const size_t off = ws.off;
            const u16 *w16 = is16(W[0]) && ff_chunked(W[0]->ptr, N, W[0]->ld) ? static_cast<const u16 *>(W[0]->ptr) : nullptr;
            const bool widen = is16(W[0]) && !w16 && M >= 8192 && K > 64 && K <= 256 && N <= 256;      // the kernel reads fp32 or whole 16-byte chunks
            float *wide = widen ? ws.get<float>((size_t)K * N) : nullptr;
            if (widen && ws.ok) {
                rc = sgnn_launch_ff_convert(ctx, view(W[0]), K, N, ff_mat{wide, N, 0}, st);
                if (rc) return rc;
            }
            if (!is16(W[0]) || w16 || (widen && ws.ok)) {
                rc = sgnn_launch_gemm_bwd(ctx, K, N, M, X->ptr, X->ld, D, ldd, widen ? wide : (w16 ? nullptr : static_cast<const float *>(W[0]->ptr)), widen ? N : W[0]->ld, dX->ptr, dX->ld,
                                          false, false, is16(dW[0]) ? nullptr : static_cast<float *>(dW[0]->ptr), nullptr, &ws, st, w16,
                                          is16(dW[0]) ? static_cast<u16 *>(dW[0]->ptr) : nullptr, dW[0]->ld);
                if (rc != SGNN_ERR_UNSUPPORTED) return rc;
            }
            ws.off = off;
            ws.ok = true;
        }
        if (any_dw) {
            const size_t off = ws.off;
            rc = operand(ctx, name, X, false, &ws, st, &x);
            if (rc) return rc;
            rc = weights(1, x, d, nullptr, nullptr);
            if (rc) return rc;
            ws.off = off;
        }
        if (!dX || dx_done) return SGNN_OK;
        rc = weight_operands();
        if (rc) return rc;
        return sgnn_launch_ff_nt(ctx, 1, M, K, N, n, d, w, nullptr, nullptr, view(dX), &ws, st);
    }
    // fp32.  One matrix of weights and few multiplications, or few columns: D as it is, both products by the kernel that splits what it reads (gemm_split.hip), the one for
    // the weights with the column sums of D; three launches fewer.  us of all kernels, parts made first / split as read, M x K x N: 100 x 256 x 256 32 / 21,
    // 1200 x 1024 x 256 58 / 47, 2500 x 256 x 256 46 / 31, 30000 x 256 x 256 98 / 88, 100000 x 64 x 64 86 / 58, 100000 x 1536 x 90 805 / 625; past the rule 2500 x 1024 x 256
    // 52 / 67, 1200 x 1024 x 1024 65 / 97, 30000 x 200 x 531 148 / 199, 10000 x 1536 x 90 94 / 98
    if (n == 1 && M >= 4 && K >= 4 && N >= 4 && ((double)M * (double)K * (double)N <= 5e8 || (K <= 256 && N <= 256) || (N <= 128 && M >= 16384))) {
        float *const sums = any_dw ? db[0] : nullptr;          // the product for the weights has them as well
        if (!is_dy || (db[0] && !any_dw)) {
            float *const none[1] = {any_dw ? nullptr : db[0]};
            rc = sgnn_launch_ff_act_bwd(ctx, M, N, np, act, view(dY), z0, nullptr, is_dy ? ff_mat{nullptr, 0, 0} : d0, nullptr, none, &ws, st);
        }
        const float *const d = static_cast<const float *>(D);
        if (!rc && any_dw)
            rc = sgnn_launch_gemm_split(ctx, 1, 0, K, N, M, static_cast<const float *>(X->ptr), X->ld, nullptr, d, ldd, nullptr, 0, static_cast<float *>(dW[0]->ptr), dW[0]->ld, nullptr, 0,
                                        sums, &ws, st);
        if (rc || !dX) return rc;
        if (few) return few_rows();
        return sgnn_launch_gemm_split(ctx, 0, 1, M, K, N, d, ldd, nullptr, static_cast<const float *>(W[0]->ptr), W[0]->ld, nullptr, 0, static_cast<float *>(dX->ptr), dX->ld, nullptr, 0,
                                      nullptr, &ws, st);
    }
    // The gradients' rows are scaled by themselves, the rows of X so that with the gradients' all products have one scale (ff_gemm.hip)
    const bool tiles_dx = dX && !few, split = any_dw || tiles_dx;
    // the gradients as parts at once where nothing else reads them and a row fits the registers
    const unsigned in_registers = split && !few && !is_dy ? sgnn_ff_act_bwd_parts_groups(M, np) : 0;
    if (!in_registers) rc = gradients();
    if (!rc && few) rc = few_rows();
    if (rc || !split) return rc;
    ff_op d[2];
    ff_parts job[3];
    ff_scan scans[2];
    int jobs = 0, nw = 0;
    int32_t *const ex_d = ws.get<int32_t>((size_t)M + 2), *const ex = ex_d + M;          // of the rows of D; of the weights, and of x d
    int32_t *ex_x = nullptr;
    uint32_t *const largest = ws.get<uint32_t>(2 * FF_SCAN_WORDS + FF_ROW_WORDS), *const key = largest + 2 * FF_SCAN_WORDS;
    d[0] = d[1] = parts_op(&ws, M, n * np);
    d[1].p += 2 * np;
    if (any_dw) {
        x = parts_op(&ws, M, K);
        ex_x = ws.get<int32_t>((size_t)M);
        job[jobs++] = ff_parts{scan(X), key, (int)(in_registers ? in_registers : sgnn_ff_row_groups(M, n * np)), ex_d, ex + 1, const_cast<u16 *>(x.p), x.ld};
    }
    for (; tiles_dx && nw < n; ++nw) {
        w[nw] = parts_op(&ws, K, N);
        scans[nw] = scan(W[nw]);
    }
    if (!ws.ok) return no_scratch(ctx, name);
    const int words = nw * (int)sgnn_ff_scan_groups(nw, scans);
    for (int q = 0; q < nw; ++q) job[jobs++] = ff_parts{scans[q], largest, words, nullptr, ex, const_cast<u16 *>(w[q].p), w[q].ld};
    const ff_scan ds = {static_cast<const float *>(D), M, n * np, ldd};
    const ff_row_parts xr = {scan(X), nullptr, 0, ex_x, nullptr, nullptr}, dr = {ds, const_cast<u16 *>(d[0].p), d[0].ld, ex_d, ex_x, any_dw ? key : nullptr};
    // the largest weights ride along with the first launch over rows
    if (any_dw) rc = sgnn_launch_ff_row_parts(ctx, xr, nw, scans, largest, st);
    if (in_registers) {
        if (!rc && !any_dw) rc = sgnn_launch_ff_row_parts(ctx, ff_row_parts{{nullptr, 0, 8, 8}, nullptr, 0, nullptr, nullptr, nullptr}, nw, scans, largest, st);
        if (!rc) rc = sgnn_launch_ff_act_bwd_parts(ctx, M, N, np, act, view(dY), z0, n == 2 ? &z1 : nullptr, dr, db, &ws, st);
    } else if (!rc) rc = sgnn_launch_ff_row_parts(ctx, dr, any_dw ? 0 : nw, scans, largest, st);
    if (!rc) rc = sgnn_launch_ff_parts(ctx, jobs, job, st);
    if (!rc && any_dw) rc = weights(2, x, d, nullptr, ex + 1);
    if (!rc && tiles_dx) rc = sgnn_launch_ff_nt(ctx, 2, M, K, N, n, d, w, ex_d, ex, view(dX), &ws, st);
    return rc;
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
    // fp32: both gradients of the pre-activations and their parts, the parts of X and of both weights; bfloat16 needs less
    size_t need = rows * (2 * dn * 8 + di * 4 + 8) + 2 * di * dn * 4 + std::max(sgnn_ff_gemm_ws_bytes(di, dn), sgnn_ff_rows_ws_bytes()) + sgnn_ff_sums_ws_bytes(dn) +
                  (2 * FF_SCAN_WORDS + FF_ROW_WORDS) * 4 + 16 * 256;
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
