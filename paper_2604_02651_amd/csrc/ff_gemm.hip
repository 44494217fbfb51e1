// Products of bfloat16 matrices of any size for the feed-forward operators, with what belongs to the operator in the epilogue:
//   linear   Y = act(A B + bias) + R                          A [M x K], B [K x N]
//   gated    Y = act(A B0 + bias0) * (A B1 + bias1)           both projections of a row and column in one wavefront
//   nt       Y = sum over s of A[s] B[s]^T                    the gradient of the input, B[s] [N x K]
//   tn       C[s] = A^T B[s], split along the rows            the gradients of the weights, A [K x M]
//
// A workgroup computes a BM x BN tile, slices of BK along the reduction staged in LDS by direct global -> LDS loads (16 bytes a lane, no registers
// in between), STAGES - 1 slices ahead, one barrier a slice.  An operand lies in LDS as it lies in memory:
//   reduction along a row (A of the first three, B of nt): BK values a row, read 16 bytes a lane;
//   reduction across the rows (B of the first two, both of tn): read by transposing LDS reads, which give a lane four reduction steps of its column.
// The 16-byte chunks of a row are swizzled by the row so that the rows which are read together lie in different banks; direct loads write LDS in lane
// order, so the swizzle is in the global address that a lane loads from.  Chunks behind the end of the reduction come from a block of zeros, rows
// and columns behind the edge of the matrix repeat the last ones and feed results that are never stored.
// v_mfma_f32_32x32x16_bf16 computes the transposed tile: register r of lane (kh, li) is row li, column 8 (r / 4) + 4 kh + r % 4 of a
// block: four adjacent columns a lane, which the epilogue brings to eight through LDS.
#include "ff.h"
#include "ff_act.h"

namespace {

// what a load behind the end of the reduction brings
__device__ const u32x4 ff_zeros = {0u, 0u, 0u, 0u};

enum { FFK_LINEAR = 0, FFK_GLU = 1, FFK_PARTIAL = 2 };

struct ffg_args {
    int64_t M, K;
    int N;                            // columns of one result matrix
    int segs, mats;                   // nt: segments of the reduction; tn: results side by side
    const u16 *A[2]; int64_t lda;
    const u16 *B[2]; int64_t ldb[2];  // of each segment, result or projection; ldb[1] of the second projection only
    ff_epilogue e;
    uint32_t mtiles, ntiles, splits;  // ntiles of one matrix
    int slices, per_split;            // slices of BK along the whole reduction, and of one range of it
    float *partial;                   // [splits][mats][M][N]
};

// Operand of R rows (or columns) by BK reduction steps in LDS
template <int R, int BK, bool TR> struct ffg_operand {
    static constexpr int ROW = TR ? R * 2 : BK * 2, LINES = TR ? BK : R, CH = ROW / 16, BYTES = R * BK * 2;
    // chunk c of line l is at c ^ swizzle(l)
    static __device__ __forceinline__ int swizzle(int l)
    {
        if constexpr (TR) return R >= 128 ? 4 * (l & 3) : 4 * ((l >> 1) & 1);
        else return BK == 64 ? (l >> 1) & 7 : (l >> 2) & 3;
    }
};

template <int BM, int BN, int WM, int WN, int BK, int STAGES, bool ATR, bool BTR, int KIND>
__global__ __launch_bounds__(64 * WM * WN, BM * BN >= 65536 ? 2 : 1) void ff_gemm_kernel(ffg_args a)
{
    // gated: the tile's columns are half of B0's, half of B1's, each an operand of its own in LDS
    constexpr int PARTS = KIND == FFK_GLU ? 2 : 1, BNP = BN / PARTS;
    using OA = ffg_operand<BM, BK, ATR>;
    using OB = ffg_operand<BNP, BK, BTR>;
    constexpr int NW = WM * WN, TM = BM / 32 / WM, TN = BN / 32 / WN, STAGE = OA::BYTES + PARTS * OB::BYTES;
    constexpr int AJ = OA::BYTES / 1024 / NW, BJ = OB::BYTES / 1024 / NW, LOADS = AJ + PARTS * BJ;
    static_assert(OA::BYTES % (1024 * NW) == 0 && OB::BYTES % (1024 * NW) == 0, "a wavefront's loads are of one operand each");
    static_assert(KIND != FFK_GLU || (TN == 2 && BTR), "a wavefront has the same columns of both projections");
    extern __shared__ __attribute__((aligned(16))) unsigned char ffg_smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 31, kh = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;

    // Workgroups are dealt to the eight XCDs in turn: each XCD takes a run of tiles, four row blocks by all columns after each other (of one range of
    // the reduction, where it is split), so that what its L2 holds is read by several of its workgroups.
    const uint32_t per_mat = a.mtiles * a.ntiles, tiles = per_mat * a.mats * a.splits, run = (tiles + 7) / 8;
    const uint32_t id = (blockIdx.x & 7) * run + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= run || id >= tiles) return;
    const uint32_t z = id / (per_mat * a.mats), t = id % (per_mat * a.mats), cols = a.ntiles * a.mats, group = t / (4 * cols);
    const uint32_t gm = min(4u, a.mtiles - 4 * group), in = t % (4 * cols);
    const uint32_t bm = 4 * group + in % gm, bc = in / gm, mat = bc / a.ntiles, bn = bc % a.ntiles;
    const int64_t m0 = (int64_t)bm * BM;
    const int n0 = (int)bn * BNP;
    const int s0 = (int)z * a.per_split, nslices = min(a.slices - s0, a.per_split), seg_slices = (int)((a.K + BK - 1) / BK);

    // A lane's place in the wave-loads of a slice: load j of an operand fills KB wave + NW j of its part.  off: bytes from the tile's first value.
    uint32_t off_a[AJ], off_b[PARTS][BJ];
    auto place = [&](auto op, int j, int &line, int &chunk) {
        using O = decltype(op);
        const int p = (wave + NW * j) * 64 + lane;
        line = p / O::CH;
        chunk = (p % O::CH) ^ O::swizzle(line);
    };
    auto offset = [&](auto op, bool tr, int j, int64_t ld, int64_t lines_left) {
        int line, c;
        place(op, j, line, c);
        const int64_t last = lines_left - 1;
        return tr ? (uint32_t)line * (uint32_t)(2 * ld) + 16u * (uint32_t)min((int64_t)c, last / 8) : (uint32_t)min((int64_t)line, last) * (uint32_t)(2 * ld) + 16u * (uint32_t)c;
    };
#pragma unroll
    for (int j = 0; j < AJ; ++j) off_a[j] = offset(OA(), ATR, j, a.lda, a.M - m0);
#pragma unroll
    for (int q = 0; q < PARTS; ++q)
#pragma unroll
        for (int j = 0; j < BJ; ++j) off_b[q][j] = offset(OB(), BTR, j, a.ldb[q], a.N - n0);
    auto issue = [&](int s) {
        const int sl = s0 + min(s, nslices - 1);        // past the end: the last slice again, into a stage nobody reads
        const int seg = a.segs > 1 && sl >= seg_slices ? 1 : 0;
        const int64_t k0 = (int64_t)(sl - seg * seg_slices) * BK;
        unsigned char *stage = ffg_smem + (s % STAGES) * STAGE + 1024 * wave;
        const int left = (int)min(a.K - k0, (int64_t)BK);
        auto part = [&](auto op, bool tr, auto &off, const u16 *first, unsigned char *to) {
            constexpr int J = sizeof(off) / sizeof(off[0]);
            const unsigned char *g = reinterpret_cast<const unsigned char *>(first);
            if (left >= BK) {
#pragma unroll
                for (int j = 0; j < J; ++j) __builtin_amdgcn_global_load_lds(STREAM_GPTR(g + off[j]), STREAM_LPTR(to + 1024 * NW * j), 16, 0, 0);
            } else {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    int line, c;
                    place(op, j, line, c);
                    const unsigned char *p = (tr ? line : 8 * c) < left ? g + off[j] : reinterpret_cast<const unsigned char *>(&ff_zeros);
                    __builtin_amdgcn_global_load_lds(STREAM_GPTR(p), STREAM_LPTR(to + 1024 * NW * j), 16, 0, 0);
                }
            }
        };
        part(OA(), ATR, off_a, a.A[seg] + (ATR ? k0 * a.lda + m0 : m0 * a.lda + k0), stage);
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            const int which = KIND == FFK_GLU ? q : (KIND == FFK_PARTIAL ? (int)mat : seg);
            part(OB(), BTR, off_b[q], a.B[which] + (BTR ? k0 * a.ldb[q] + n0 : (int64_t)n0 * a.ldb[q] + k0), stage + OA::BYTES + q * OB::BYTES);
        }
    };

    // where a lane reads its operands: blocks of 32 rows / columns
    const int x = lane & 15, r3 = x >> 2, half = (lane >> 4) & 1;
    auto tr_at = [&](auto op, int blk) {
        using O = decltype(op);
        return (8 * kh + r3) * O::ROW + ((blk * 4 + 2 * half + ((x & 3) >> 1)) ^ O::swizzle(r3)) * 16 + (x & 1) * 8;
    };
    auto kc_at = [&](auto op, int blk) {
        using O = decltype(op);
        return (32 * blk + li) * O::ROW + ((kh ^ O::swizzle(li)) * 16);
    };
    int at_a[TM], at_b[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) at_a[i] = ATR ? tr_at(OA(), wm * TM + i) : kc_at(OA(), wm * TM + i);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int blk = KIND == FFK_GLU ? wn : wn * TN + j;
        at_b[j] = OA::BYTES + (KIND == FFK_GLU ? j * OB::BYTES : 0) + (BTR ? tr_at(OB(), blk) : kc_at(OB(), blk));
    }

    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(s);
    for (int s = 0; s < nslices; ++s) {
        STREAM_WAIT_VMCNT((STAGES - 2) * LOADS);         // slice s has landed (this wavefront's part); the later ones may be in flight
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();                    // everybody's part has; and everybody is through slice s - 1
        asm volatile("" ::: "memory");
        issue(s + STAGES - 1);                           // into the stage slice s - 1 was read from
        const unsigned char *stage = ffg_smem + (s % STAGES) * STAGE;
#pragma unroll
        for (int ks = 0; ks < BK / 16; ++ks) {
            bf16x8 fa[TM], fb[TN];
            auto fetch = [&](auto op, bool tr, int at) {
                using O = decltype(op);
                if (tr) {
                    const uint2 lo = read_tr(stage + at + 16 * ks * O::ROW), hi = read_tr(stage + at + (16 * ks + 4) * O::ROW);
                    return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
                }
                return read_row(stage + (at ^ (32 * ks)));
            };
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = fetch(OB(), BTR, at_b[j]);
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = fetch(OA(), ATR, at_a[i]);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
        }
    }
    STREAM_WAIT_VMCNT(0);       // the repeated loads past the end are still in flight: nothing may leave before they land

    // A wavefront's blocks go through a strip of LDS of its own, 32 rows at a time, so that a lane has eight adjacent columns and rows leave (and the
    // residual is read) in pieces of 64 bytes and more.
    constexpr int WC = 32 * TN, LDW = WC + 4, EC = KIND == FFK_GLU ? WC / 2 : WC, LPR = EC / 8, RPS = 64 / LPR;
    static_assert(NW * 32 * LDW * 4 <= STAGES * STAGE, "the strips fit where the slices were");
    float *const strip = reinterpret_cast<float *>(ffg_smem) + wave * 32 * LDW;
    __builtin_amdgcn_s_barrier();                            // everybody is through the last slice
    asm volatile("" ::: "memory");
    const ff_epilogue &ep = a.e;
    const int c = 8 * (lane % LPR), col = n0 + EC * wn + c, cols_left = a.N - col;
    float b0[8], b1[8];
    if constexpr (KIND != FFK_PARTIAL) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            b0[e] = ep.bias[0] ? ep.bias[0][min(col + e, a.N - 1)] : 0.f;
            b1[e] = KIND == FFK_GLU && ep.bias[1] ? ep.bias[1][min(col + e, a.N - 1)] : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4 *>(strip + li * LDW + 32 * j + 8 * q + 4 * kh) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
#pragma unroll 1
        for (int r0 = 0; r0 < 32; r0 += RPS) {
            const int r = r0 + lane / LPR;
            const int64_t row = m0 + 32 * (wm * TM + i) + r;
            if (row >= a.M || cols_left <= 0) continue;
            const float *at = strip + r * LDW + c;
            float v[8], u[8];
            auto read = [&](float (&x)[8], int from) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 w = *reinterpret_cast<const f32x4 *>(at + from + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[4 * h + e] = w[e];
                }
            };
            read(v, 0);
            if constexpr (KIND == FFK_PARTIAL) {
                const ff_mat o = {a.partial + ((int64_t)z * a.mats + mat) * a.M * a.N, a.N, 0};
                ff_store<FF_T32, 8>(v, o, row, col, cols_left);
            } else {
                if (KIND == FFK_GLU) read(u, EC);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] += b0[e];
                    if (KIND == FFK_GLU) u[e] += b1[e];
                }
                if (ep.Z[0].p) ff_store<FF_TANY, 8>(v, ep.Z[0], row, col, cols_left);
                if (KIND == FFK_GLU && ep.Z[1].p) ff_store<FF_TANY, 8>(u, ep.Z[1], row, col, cols_left);
                if (KIND == FFK_LINEAR && ep.R.p) ff_load<FF_TANY, 8>(u, ep.R, row, col, cols_left);
                ff_with_act(ep.act, [&](auto act) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = ff_act<decltype(act)::value>(v[e]);
                });
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = KIND == FFK_GLU ? v[e] * u[e] : (ep.R.p ? v[e] + u[e] : v[e]);
                ff_store<FF_TANY, 8>(v, ep.Y, row, col, cols_left);
            }
        }
    }
}

// C[s] = sum over the ranges of partial[range][s], in their order
__global__ __launch_bounds__(256) void ff_reduce_kernel(const float *__restrict__ partial, int splits, int mats, int64_t M, int N, ff_mat C0, ff_mat C1)
{
    const int chunks = (N + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = M * chunks;
    if (i >= n * mats) return;
    const int mat = (int)(i / n);
    const int64_t row = (i % n) / chunks;
    const int col = 4 * (int)(i % chunks), left = N - col;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int z = 0; z < splits; ++z) {
        float v[4];
        ff_load<FF_T32, 4>(v, ff_mat{partial + ((int64_t)z * mats + mat) * M * N, N, 0}, row, col, left);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
    ff_store<FF_TANY, 4>(s, mat ? C1 : C0, row, col, left);
}

template <int BM, int BN, int WM, int WN, int BK, int STAGES, bool ATR, bool BTR, int KIND> int launch(sgnn_ctx *ctx, ffg_args a, int64_t per_split, hipStream_t st)
{
    constexpr int LDS = STAGES * (BM + BN) * BK * 2;
    a.mtiles = cdiv(a.M, BM);
    a.ntiles = cdiv(a.N, KIND == FFK_GLU ? BN / 2 : BN);
    const int64_t slices = (int64_t)a.segs * cdiv(a.K, BK);
    a.slices = (int)slices;
    a.per_split = KIND == FFK_PARTIAL ? (int)per_split : (int)slices;
    a.splits = cdiv(slices, a.per_split);
    const uint64_t tiles = (uint64_t)a.mtiles * a.ntiles * a.mats * a.splits;
    if (tiles > 0x70000000ull || slices > 0x7fffffff) return sgnn_fail(ctx, SGNN_ERR_UNSUPPORTED, "feed-forward product: more than 2^31 tiles");
    SGNN_HIP(ctx, (sgnn_allow_lds<&ff_gemm_kernel<BM, BN, WM, WN, BK, STAGES, ATR, BTR, KIND>>(ctx, LDS)));
    char tag[56] = "";
    if (ctx->prof_on) snprintf(tag, sizeof(tag), "%c%c%s %dx%d %lldx%dx%lld", ATR ? 'T' : 'N', BTR ? 'N' : 'T', KIND == FFK_GLU ? " gated" : "", BM, BN, (long long)a.M, a.N, (long long)a.K);
    SGNN_LAUNCH(ctx, st, "ff_gemm_kernel", tag, (ff_gemm_kernel<BM, BN, WM, WN, BK, STAGES, ATR, BTR, KIND>), dim3((unsigned)((tiles + 7) / 8 * 8)),
                dim3(64 * WM * WN), LDS, st, a);
    return SGNN_OK;
}

} // namespace

int sgnn_launch_ff_linear(sgnn_ctx *ctx, int64_t M, int64_t N, int64_t K, const u16 *A, int64_t lda, const u16 *B, int64_t ldb, const ff_epilogue &e,
                          hipStream_t st)
{
    ffg_args a = {};
    a.M = M; a.N = (int)N; a.K = K; a.segs = a.mats = 1;
    a.A[0] = A; a.lda = lda; a.B[0] = B; a.ldb[0] = ldb; a.e = e;
    return launch<128, 128, 2, 2, 64, 2, false, true, FFK_LINEAR>(ctx, a, 0, st);
}

int sgnn_launch_ff_glu(sgnn_ctx *ctx, int64_t M, int64_t N, int64_t K, const u16 *A, int64_t lda, const u16 *B0, int64_t ldb0, const u16 *B1, int64_t ldb1,
                       const ff_epilogue &e, hipStream_t st)
{
    ffg_args a = {};
    a.M = M; a.N = (int)N; a.K = K; a.segs = a.mats = 1;
    a.A[0] = A; a.lda = lda; a.B[0] = B0; a.ldb[0] = ldb0; a.B[1] = B1; a.ldb[1] = ldb1; a.e = e;
    return launch<128, 128, 2, 2, 64, 2, false, true, FFK_GLU>(ctx, a, 0, st);
}

int sgnn_launch_ff_nt(sgnn_ctx *ctx, int64_t M, int64_t N, int64_t K, int segs, const u16 *const *A, int64_t lda, const u16 *const *B, int64_t ldb,
                      const ff_mat &Y, hipStream_t st)
{
    ffg_args a = {};
    a.M = M; a.N = (int)N; a.K = K; a.segs = segs; a.mats = 1;
    a.lda = lda;
    for (int s = 0; s < segs; ++s) { a.A[s] = A[s]; a.B[s] = B[s]; a.ldb[s] = ldb; }
    a.e.act = SGNN_ACT_NONE;
    a.e.Y = Y;
    return launch<128, 128, 2, 2, 64, 2, false, false, FFK_LINEAR>(ctx, a, 0, st);
}

size_t sgnn_ff_tn_ws_bytes(uint64_t rows, uint64_t d_in, uint64_t d_out)
{
    return 2 * 32 * d_in * d_out * 4 + 256;
}

int sgnn_launch_ff_tn(sgnn_ctx *ctx, int64_t M, int64_t N, int64_t K, int mats, const u16 *A, int64_t lda, const u16 *const *B, int64_t ldb, const ff_mat *C,
                      ws_alloc *ws, hipStream_t st)
{
    ffg_args a = {};
    a.M = M; a.N = (int)N; a.K = K; a.segs = 1; a.mats = mats;
    a.A[0] = A; a.lda = lda;
    for (int s = 0; s < mats; ++s) { a.B[s] = B[s]; a.ldb[s] = ldb; }
    const int64_t slices = cdiv(K, 64), tiles = (int64_t)cdiv(M, 128) * cdiv(N, 128) * mats;
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(32, slices / 4), 512 / tiles));
    const int64_t per = cdiv(slices, splits);
    const size_t off = ws->off;
    a.partial = ws->get<float>((size_t)cdiv(slices, per) * mats * M * N);
    if (!ws->ok) return sgnn_fail(ctx, SGNN_ERR_CAPACITY, "feed-forward operator: scratch too small: call sgnn_ctx_reserve_ffn");
    const int rc = launch<128, 128, 2, 2, 64, 2, true, true, FFK_PARTIAL>(ctx, a, per, st);
    if (rc) return rc;
    SGNN_LAUNCH(ctx, st, "ff_reduce_kernel", SGNN_TAG, ff_reduce_kernel, dim3(cdiv(M * ((N + 3) / 4) * mats, 256)), dim3(256), 0, st, a.partial,
                (int)cdiv(slices, per), mats, M, (int)N, C[0], C[mats - 1]);
    ws->off = off;         // what the caller launches next on this stream may have the scratch
    return SGNN_OK;
}
