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
//
// fp32 products take the same path on the fp16 pipe.  Values are scaled by powers of two, the largest magnitude of a row (of X, of the gradients) or of
// a weight matrix to [2^14, 2^15), and every one is split into two fp16 parts (ff_elem.hip):
//   x = x1 + 2^-11 x2,  x1 = fp16(x), x2 = fp16(2^11 (x - x1)),  |error| <= 2^-23 |x|
//   a b = a1 b1 + 2^-11 (a1 b2 + a2 b1) + up to 2^-21 |a b| (the product of the second parts, and what the parts leave out)
// three products of exact terms, the leading ones and the others in accumulators of their own.  The method is that of Ootomo and Yokota, "Recovering
// single precision accuracy from Tensor Cores while surpassing the FP32 theoretical peak performance" (2022).  The second part's own scale keeps all of
// its bits down to 2^-29 of the largest value; smaller values are off by up to 2^-51 of it.  For tn, where the reduction is along the rows, row m of X is
// scaled so that all of x d have one scale: the largest products keep their bits, rows that add nothing count for nothing.  An infinity or NaN is its
// own first part with a second part of 0, and a sum of first parts that is not finite is the result.
#include "ff.h"
#include "ff_act.h"

namespace {

// what a load behind the end of the reduction brings
__device__ const u32x4 ff_zeros = {0u, 0u, 0u, 0u};

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

enum { FFK_LINEAR = 0, FFK_GLU = 1, FFK_PARTIAL = 2 };

struct ffg_args {
    int64_t M, K;
    int N;                            // columns of one result matrix
    int segs, mats;                   // nt: segments of the reduction; tn: results side by side
    ff_op A[2], B[2];                 // A of each segment, B of each segment, result or projection (of the first two one leading dimension)
    const int32_t *ex_rows, *ex;      // fp32: the exponents by which the rows of A (or null) and everything else were scaled
    ff_epilogue e;
    uint32_t mtiles, ntiles, splits;  // ntiles of one matrix
    int slices, per_split;            // slices of BK along the whole reduction, and of one range of it
    float *partial;                   // tn: [splits][mats][M][N]; else, where the reduction is split: [tiles][splits][BM BN]
    uint32_t *arrived;                // [tiles], zero between calls
};

// Operand of R rows (or columns) by BK reduction steps in LDS.  PL = 2: the 16-byte chunks of the two parts alternate in a row.
template <int PL, int R, int BK, bool TR> struct ffg_operand {
    static constexpr int ROW = (TR ? R : BK) * 2 * PL, CH = ROW / 16, BYTES = R * BK * 2 * PL;
    // Chunk c of line l is at c ^ swizzle(l): what is read together, chunks of 32 bytes (of one part: every other 16) of four rows with transposing reads, one chunk of
    // sixteen rows without, lies in different banks of the 256 bytes.
    static __device__ __forceinline__ int swizzle(int l)
    {
        if constexpr (TR) return PL == 2 ? (l & 1) | ((l >> 1) & 1) << 3 : (R >= 128 ? 4 * (l & 3) : 4 * ((l >> 1) & 1));
        else return ROW == 128 ? (l >> 1) & 7 : (l >> 2) & 3;
    }
};

// PL: 1 bfloat16, 2 fp32 as two fp16 parts
template <int PL, int BM, int BN, int WM, int WN, int BK, int STAGES, bool ATR, bool BTR, int KIND>
__global__ __launch_bounds__(64 * WM * WN, BM * BN * PL >= 32768 ? 2 : 1) void ff_gemm_kernel(ffg_args a)
{
    // gated: the tile's columns are half of B0's, half of B1's, each an operand of its own in LDS
    constexpr int PARTS = KIND == FFK_GLU ? 2 : 1, BNP = BN / PARTS;
    using OA = ffg_operand<PL, BM, BK, ATR>;
    using OB = ffg_operand<PL, BNP, BK, BTR>;
    // a slice in LDS: A, then B, or the tile's columns of both; loads of 1 KB (a wavefront's), load l of the slice by wavefront l % NW
    constexpr int NW = WM * WN, TM = BM / 32 / WM, TN = BN / 32 / WN, STAGE = OA::BYTES + PARTS * OB::BYTES;
    constexpr int AL = OA::BYTES / 1024, BL = OB::BYTES / 1024, LOADS = STAGE / 1024 / NW;
    constexpr bool EVEN = AL % NW == 0 && BL % NW == 0;         // which operand a load is of does not depend on the wavefront
    static_assert(OA::BYTES % 1024 == 0 && OB::BYTES % 1024 == 0 && STAGE % (1024 * NW) == 0, "whole loads, as many for every wavefront");
    static_assert(KIND != FFK_GLU || (TN % 2 == 0 && BTR), "a wavefront has the same columns of both projections");
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

    // load j of the wavefront: of which part of the slice, and the lane's place in it
    struct place { bool b; int q, line, chunk; };
    auto where = [&](int j) {
        const int l = (EVEN ? 0 : wave) + NW * j;
        place p;
        p.b = l >= AL;
        p.q = p.b ? (l - AL) / BL : 0;
        const int at = ((p.b ? (l - AL) % BL : l) + (EVEN ? wave : 0)) * 64 + lane;
        p.line = p.b ? at / OB::CH : at / OA::CH;
        p.chunk = p.b ? (at % OB::CH) ^ OB::swizzle(p.line) : (at % OA::CH) ^ OA::swizzle(p.line);
        return p;
    };
    uint32_t off[LOADS];          // bytes from the tile's first value
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const place p = where(j);
        const bool tr = p.b ? BTR : ATR;
        const int64_t last = p.b ? a.N - 1 - n0 : a.M - 1 - m0, ld = p.b ? a.B[KIND == FFK_GLU ? p.q : 0].ld : a.A[0].ld;
        off[j] = tr ? (uint32_t)p.line * (uint32_t)(2 * ld) + 16u * (uint32_t)(PL * min((int64_t)(p.chunk / PL), last / 8) + p.chunk % PL)
                    : (uint32_t)min((int64_t)p.line, last) * (uint32_t)(2 * ld) + 16u * (uint32_t)p.chunk;
    }
    auto issue = [&](int s) {
        const int sl = s0 + min(s, nslices - 1);        // past the end: the last slice again, into a stage nobody reads
        const int seg = a.segs > 1 && sl >= seg_slices ? 1 : 0;
        const int64_t k0 = (int64_t)(sl - seg * seg_slices) * BK;
        unsigned char *stage = ffg_smem + (s % STAGES) * STAGE + 1024 * wave;
        const int left = (int)min(a.K - k0, (int64_t)BK);
        const u16 *first_a = a.A[seg].p + (ATR ? k0 * a.A[0].ld + PL * m0 : m0 * a.A[0].ld + PL * k0);
        const u16 *first_b[PARTS];
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            const int which = KIND == FFK_GLU ? q : (KIND == FFK_PARTIAL ? (int)mat : seg);
            const int64_t ld = a.B[KIND == FFK_GLU ? q : 0].ld;
            first_b[q] = a.B[which].p + (BTR ? k0 * ld + PL * n0 : (int64_t)n0 * ld + PL * k0);
        }
        auto base = [&](const place &p) { return reinterpret_cast<const unsigned char *>(p.b ? first_b[PARTS > 1 ? p.q : 0] : first_a); };
        if (left >= BK) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) __builtin_amdgcn_global_load_lds(STREAM_GPTR(base(where(j)) + off[j]), STREAM_LPTR(stage + 1024 * NW * j), 16, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const place p = where(j);
                const unsigned char *g = ((p.b ? BTR : ATR) ? p.line : 8 * (p.chunk / PL)) < left ? base(p) + off[j] : reinterpret_cast<const unsigned char *>(&ff_zeros);
                __builtin_amdgcn_global_load_lds(STREAM_GPTR(g), STREAM_LPTR(stage + 1024 * NW * j), 16, 0, 0);
            }
        }
    };

    // where a lane reads its operands: blocks of 32 rows / columns
    const int x = lane & 15, r3 = x >> 2, half = (lane >> 4) & 1;
    auto tr_at = [&](auto op, int blk) {
        using O = decltype(op);
        return (8 * kh + r3) * O::ROW + ((PL * (blk * 4 + 2 * half + ((x & 3) >> 1))) ^ O::swizzle(r3)) * 16 + (x & 1) * 8;
    };
    auto kc_at = [&](auto op, int blk) {
        using O = decltype(op);
        return (32 * blk + li) * O::ROW + ((PL * kh) ^ O::swizzle(li)) * 16;
    };
    int at_a[TM], at_b[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) at_a[i] = ATR ? tr_at(OA(), wm * TM + i) : kc_at(OA(), wm * TM + i);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int blk = KIND == FFK_GLU ? wn * (TN / 2) + j % (TN / 2) : wn * TN + j;
        at_b[j] = OA::BYTES + (KIND == FFK_GLU ? j / (TN / 2) * OB::BYTES : 0) + (BTR ? tr_at(OB(), blk) : kc_at(OB(), blk));
    }

    f32x16 acc[TM][TN], low[PL > 1 ? TM : 1][PL > 1 ? TN : 1];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                acc[i][j][r] = 0.f;
                if (PL > 1) low[PL > 1 ? i : 0][PL > 1 ? j : 0][r] = 0.f;
            }

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
            u32x4 fa[PL][TM], fb[PL][TN];
            auto fetch = [&](auto op, bool tr, int at, int part) {
                using O = decltype(op);
                if (tr) {
                    at ^= 16 * part;
                    const uint2 lo = read_tr(stage + at + 16 * ks * O::ROW), hi = read_tr(stage + at + (16 * ks + 4) * O::ROW);
                    return u32x4{lo.x, lo.y, hi.x, hi.y};
                }
                return read_row(stage + (at ^ (32 * PL * ks + 16 * part)));
            };
#pragma unroll
            for (int p = 0; p < PL; ++p) {
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[p][j] = fetch(OB(), BTR, at_b[j], p);
#pragma unroll
                for (int i = 0; i < TM; ++i) fa[p][i] = fetch(OA(), ATR, at_a[i], p);
            }
            auto multiply = [&](auto &c, int pa, int pb) {
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        if constexpr (PL > 1) c[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, fb[pb][j]), __builtin_bit_cast(f16x8, fa[pa][i]), c[i][j], 0, 0, 0);
                        else c[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fb[pb][j]), __builtin_bit_cast(bf16x8, fa[pa][i]), c[i][j], 0, 0, 0);
                    }
            };
            multiply(acc, 0, 0);
            if constexpr (PL > 1) {
                multiply(low, 1, 0);
                multiply(low, 0, 1);
            }
        }
    }
    STREAM_WAIT_VMCNT(0);       // the repeated loads past the end are still in flight: nothing may leave before they land
    if constexpr (PL > 1) {
        const int ex = *a.ex;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t row = m0 + 32 * (wm * TM + i) + li;
            const int back = -(a.ex_rows && row < a.M ? ex + a.ex_rows[row] : ex);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float h = acc[i][j][r];
                    acc[i][j][r] = __builtin_amdgcn_ldexpf(fabsf(h) < __builtin_inff() ? fmaf(low[i][j][r], 0x1p-11f, h) : h, back);
                }
        }
    }
    if constexpr (KIND != FFK_PARTIAL) {
        if (a.splits > 1) {
            // every range leaves its sums, past the XCD's own L2; the workgroup that arrives last adds them up in their order and goes on
            __shared__ uint32_t last;
            float *const to = a.partial + ((size_t)t * a.splits + z) * (BM * BN) + wave * (TM * TN * 1024) + lane;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) __hip_atomic_store(to + ((i * TN + j) * 16 + r) * 64, acc[i][j][r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            STREAM_WAIT_VMCNT(0);
            __syncthreads();
            if (threadIdx.x == 0) {
                last = __hip_atomic_fetch_add(a.arrived + t, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (last == a.splits - 1) __hip_atomic_store(a.arrived + t, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (last != a.splits - 1) return;
            const float *const from = a.partial + (size_t)t * a.splits * (BM * BN) + wave * (TM * TN * 1024) + lane;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    // four ranges are requested together
                    f32x16 sum;
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum[r] = 0.f;
                    for (uint32_t y0 = 0; y0 < a.splits; y0 += 4) {
                        float v[4][16];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                v[u][r] = __hip_atomic_load(from + (size_t)min(y0 + u, a.splits - 1) * (BM * BN) + ((i * TN + j) * 16 + r) * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int r = 0; r < 16; ++r) sum[r] += y0 + u < a.splits ? v[u][r] : 0.f;
                    }
                    acc[i][j] = sum;
                }
        }
    }

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
                if (a.splits == 1) ff_store<FF_TANY, 8>(v, mat ? ep.Z[0] : ep.Y, row, col, cols_left);
                else ff_store<FF_T32, 8>(v, ff_mat{a.partial + ((int64_t)z * a.mats + mat) * a.M * a.N, a.N, 0}, row, col, cols_left);
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
                    for (int e = 0; e < 8; ++e) v[e] = ff_act<decltype(act)::value, PL == 1>(v[e]);
                });
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = KIND == FFK_GLU ? v[e] * u[e] : (ep.R.p ? v[e] + u[e] : v[e]);
                ff_store<FF_TANY, 8>(v, ep.Y, row, col, cols_left);
            }
        }
    }
}

// C[s] = sum over the ranges of partial[range][s]: ZL interleaved chains (the more, the fewer elements there are), then the chains in order
template <int ZL> __global__ __launch_bounds__(256) void ff_reduce_kernel(const float *__restrict__ partial, int splits, int mats, int64_t M, int N, ff_mat C0, ff_mat C1)
{
    __shared__ f32x4 red[ZL > 1 ? 256 : 1];
    const int chunks = (N + 3) / 4, zl = threadIdx.x / (256 / ZL);
    const int64_t i = (int64_t)blockIdx.x * (256 / ZL) + threadIdx.x % (256 / ZL), n = M * chunks;
    const bool in = i < n * mats;
    const int mat = in ? (int)(i / n) : 0;
    const int64_t row = in ? (i % n) / chunks : 0;
    const int col = in ? 4 * (int)(i % chunks) : 0, left = N - col;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (in) {
#pragma unroll 8
        for (int z = zl; z < splits; z += ZL) {
            float v[4];
            ff_load<FF_T32, 4>(v, ff_mat{partial + ((int64_t)z * mats + mat) * M * N, N, 0}, row, col, left);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += v[e];
        }
    }
    if constexpr (ZL > 1) {
        red[threadIdx.x] = s;
        __syncthreads();
        if (zl) return;
#pragma unroll
        for (int q = 1; q < ZL; ++q) s += red[q * (256 / ZL) + threadIdx.x];
    }
    const float v[4] = {s[0], s[1], s[2], s[3]};
    if (in) ff_store<FF_TANY, 4>(v, mat ? C1 : C0, row, col, left);
}

template <int PL, int BM, int BN, int WM, int WN, int BK, int STAGES, bool ATR, bool BTR, int KIND> int launch(sgnn_ctx *ctx, ffg_args a, int64_t splits, ws_alloc *ws, hipStream_t st)
{
    constexpr int LDS = STAGES * PL * (BM + BN) * BK * 2;
    a.mtiles = cdiv(a.M, BM);
    a.ntiles = cdiv(a.N, KIND == FFK_GLU ? BN / 2 : BN);
    const int64_t slices = (int64_t)a.segs * cdiv(a.K, BK);
    a.slices = (int)slices;
    a.per_split = (int)cdiv(slices, splits);
    a.splits = cdiv(slices, a.per_split);
    const uint64_t tiles = (uint64_t)a.mtiles * a.ntiles * a.mats * a.splits;
    if (tiles > 0x70000000ull || slices > 0x7fffffff) return sgnn_fail(ctx, SGNN_ERR_UNSUPPORTED, "feed-forward product: more than 2^31 tiles");
    const bool joined = KIND != FFK_PARTIAL && a.splits > 1;
    if (a.splits > 1) {
        a.partial = ws->get<float>(KIND == FFK_PARTIAL ? (size_t)a.splits * a.mats * a.M * a.N : tiles * BM * BN);
        if (!ws->ok) return sgnn_fail(ctx, SGNN_ERR_CAPACITY, "feed-forward operator: scratch too small: call sgnn_ctx_reserve_ffn");
    }
    if (joined) {
        a.arrived = sgnn_ff_arrived(ctx);
        const int rc = sgnn_ff_open(ctx, st);
        if (rc) return rc;
    }
    SGNN_HIP(ctx, (sgnn_allow_lds<&ff_gemm_kernel<PL, BM, BN, WM, WN, BK, STAGES, ATR, BTR, KIND>>(ctx, LDS)));
    char tag[56] = "";
    if (ctx->prof_on)
        snprintf(tag, sizeof(tag), "%c%c%s %dx%d %lldx%dx%lld%s /%u", ATR ? 'T' : 'N', BTR ? 'N' : 'T', KIND == FFK_GLU ? " gated" : "", BM, BN, (long long)a.M, a.N,
                 (long long)a.K, PL > 1 ? " f32" : "", a.splits);
    auto go = [&]() -> int {
        SGNN_LAUNCH(ctx, st, "ff_gemm_kernel", tag, (ff_gemm_kernel<PL, BM, BN, WM, WN, BK, STAGES, ATR, BTR, KIND>), dim3((unsigned)((tiles + 7) / 8 * 8)),
                    dim3(64 * WM * WN), LDS, st, a);
        return SGNN_OK;
    };
    int rc = go();
    if (joined) rc = sgnn_ff_close(ctx, rc, st);
    return rc;
}

// Tiles, by how many of them a compute unit has at a time (in LDS):
//   WIDE   bfloat16 256 x 256, fp32 256 x 128, one;   TALL   bfloat16 256 x 128, two;   MID   128 x 128, two;   SMALL   64 x 128, two
enum { FFT_WIDE, FFT_TALL, FFT_MID, FFT_SMALL };

// Tile for a result of M x N (both projections counted) and K steps of the reduction, and the ranges that is split into.
// The wide tile reads the least of LDS a product, but is alone on its compute unit: nothing runs while it fills its pipeline and writes its result.  bfloat16, us WIDE /
// TALL / MID: 8192 x 8192 x 8192 920 / 1123 / 1196, 131072 x 256 x 1408 116 / 149 / 145, 65536 x 1024 x 512 99 / 101 / 115; 262144 x 256 x 256 78 / 74 / 80, gated
// 131072 x 2 x 704 x 256 192 / 162 / 184.  fp32, WIDE / MID: 4096 x 4096 x 4096 375 / 401, 16384 x 1024 x 2048 194 / 197, 65536 x 1024 x 512 279 / 251,
// gated 32768 x 2 x 704 x 256 108 / 94.  Where the last round of wide tiles leaves most compute units idle, smaller ones are better: 16384 x 512 x 512, 128 tiles, 27 / 22 / 19.
// Fewer middle tiles than compute units: 2048 x 1024 x 2048 MID / SMALL bfloat16 27 / 23, fp32 54 / 42; with as many, 4096 x 1024 x 1024, 18.2 / 18.4, 34.6 / 35.2.
int tile_for(int pl, int64_t M, int64_t N, int64_t K, int64_t *splits)
{
    auto tiles = [&](int64_t bm, int64_t bn) { return (int64_t)cdiv(M, bm) * cdiv(N, bn); };
    *splits = 1;
    const int64_t mid = tiles(128, 128);
    if (pl == 1) {
        // rounds of tiles, a round of wide ones as the unit
        const int64_t wide = cdiv(tiles(256, 256), 256) * 6, middle = cdiv(mid, 512) * 4;
        if (K >= 512 ? wide <= middle && tiles(256, 256) >= 128 : tiles(256, 256) >= 256) return K >= 512 ? FFT_WIDE : FFT_TALL;
    } else if (K >= 2048 && tiles(256, 128) >= 256) return FFT_WIDE;
    if (mid >= 256) return FFT_MID;
    const int64_t n = tiles(64, 128), slices = cdiv(K, pl == 1 ? 64 : 32);
    // Ranges: up to a workgroup a compute unit, or two where its part is longer than 20 slices: what more of them save is 0.3 us a slice (fp32 0.6), the join costs 4.
    // us with up to 512 / 256 workgroups, bfloat16: 2500 x 1024 x 256 17.8 / 14.0, 512 x 1024 x 2 x 1024 18.7 / 15.0, 1100 x 4096 x 512 21.2 / 22.2, 2500 x 4096 x 512
    // 27 / 40; fp32 2500 x 256 x 2 x 256 24.4 / 18.5, 200 x 2048 x 2048 42.6 / 38.5, 512 x 2048 x 2048 42.6 / 44.9, 1100 x 1024 x 1024 32 / 37.
    if (n <= SGNN_FFN_COUNTS) {
        *splits = std::max<int64_t>(1, std::min<int64_t>(256 / n, slices / 4));
        if (slices > 20 * *splits) *splits = std::max<int64_t>(1, std::min<int64_t>(512 / n, slices / 4));
    }
    return FFT_SMALL;
}

template <bool ATR, bool BTR, int KIND> int launch_tile(sgnn_ctx *ctx, int pl, const ffg_args &a, int tile, int64_t splits, ws_alloc *ws, hipStream_t st)
{
    if (pl == 1) {
        if (tile == FFT_WIDE) return launch<1, 256, 256, 2, 4, 64, 2, ATR, BTR, KIND>(ctx, a, splits, ws, st);
        if constexpr (KIND != FFK_PARTIAL) {
            if (tile == FFT_TALL) return launch<1, 256, 128, 2, 2, 32, 3, ATR, BTR, KIND>(ctx, a, splits, ws, st);
        }
        if (tile == FFT_MID) return launch<1, 128, 128, 2, 2, 64, 2, ATR, BTR, KIND>(ctx, a, splits, ws, st);
        return launch<1, 64, 128, 2, 2, 64, 3, ATR, BTR, KIND>(ctx, a, splits, ws, st);
    }
    if constexpr (KIND != FFK_PARTIAL) {
        if (tile == FFT_WIDE) return launch<2, 256, 128, 4, 2, 32, 2, ATR, BTR, KIND>(ctx, a, splits, ws, st);
    }
    if (tile == FFT_MID) return launch<2, 128, 128, 2, 2, 32, 2, ATR, BTR, KIND>(ctx, a, splits, ws, st);
    return launch<2, 64, 128, 2, 2, 32, 3, ATR, BTR, KIND>(ctx, a, splits, ws, st);
}

ffg_args args(int64_t M, int64_t N, int64_t K, const int32_t *ex_rows, const int32_t *ex)
{
    ffg_args a = {};
    a.M = M; a.N = (int)N; a.K = K; a.segs = a.mats = 1;
    a.ex_rows = ex_rows; a.ex = ex;
    a.e.act = SGNN_ACT_NONE;
    return a;
}

} // namespace

int sgnn_launch_ff_nn(sgnn_ctx *ctx, int pl, int64_t M, int64_t N, int64_t K, int mats, const ff_op &A, const ff_op *B, const int32_t *ex_rows, const int32_t *ex,
                      const ff_epilogue &e, ws_alloc *ws, hipStream_t st)
{
    ffg_args a = args(M, N, K, ex_rows, ex);
    a.A[0] = a.A[1] = A;
    a.B[0] = B[0];
    a.B[1] = B[mats - 1];
    a.e = e;
    int64_t splits;
    const int tile = tile_for(pl, M, mats * N, K, &splits);
    const size_t off = ws->off;
    const int rc = mats == 2 ? launch_tile<false, true, FFK_GLU>(ctx, pl, a, tile, splits, ws, st) : launch_tile<false, true, FFK_LINEAR>(ctx, pl, a, tile, splits, ws, st);
    ws->off = off;         // what the caller launches next on this stream may have the scratch
    return rc;
}

int sgnn_launch_ff_nt(sgnn_ctx *ctx, int pl, int64_t M, int64_t N, int64_t K, int segs, const ff_op *A, const ff_op *B, const int32_t *ex_rows, const int32_t *ex,
                      const ff_mat &Y, ws_alloc *ws, hipStream_t st)
{
    ffg_args a = args(M, N, K, ex_rows, ex);
    a.segs = segs;
    for (int s = 0; s < segs; ++s) { a.A[s] = A[s]; a.B[s] = B[s]; }
    a.e.Y = Y;
    int64_t splits;
    const int tile = tile_for(pl, M, N, segs * K, &splits);
    const size_t off = ws->off;
    const int rc = launch_tile<false, false, FFK_LINEAR>(ctx, pl, a, tile, splits, ws, st);
    ws->off = off;
    return rc;
}

// Scratch of the products: partial results of tn (at most 512 ranges; over all of them 512 tiles of 128 x 128, or as many elements in others, or one result), sums of
// split tiles (512 of 64 x 128); of gemm_split.hip 768 tiles of up to 256 x 128 and the column sums that ride along
size_t sgnn_ff_gemm_ws_bytes(uint64_t d_in, uint64_t d_out)
{
    const uint64_t results = 2 * d_in * d_out;
    return std::max<uint64_t>(std::min<uint64_t>(512 * results, std::max<uint64_t>(768ull * 32768 + (1 << 18), results)), 512ull * 64 * 128) * 4 + 512;
}

int sgnn_launch_ff_tn(sgnn_ctx *ctx, int pl, int64_t M, int64_t N, int64_t K, int mats, const ff_op &A, const ff_op *B, const int32_t *ex_rows, const int32_t *ex,
                      const ff_mat *C, ws_alloc *ws, hipStream_t st)
{
    ffg_args a = args(M, N, K, ex_rows, ex);
    a.mats = mats;
    a.A[0] = a.A[1] = A;
    for (int s = 0; s < mats; ++s) a.B[s] = B[s];
    a.e.Y = C[0];             // where the reduction is not split
    a.e.Z[0] = C[mats - 1];
    const int bk = pl == 1 ? 64 : 32;
    const int64_t slices = cdiv(K, bk);
    // The wide tile for long reductions, us WIDE / MID: bfloat16 256 x 1408 x 131072 120 / 130, 1024 x 1024 x 8192 37 / 26; fp32 256 x 1408 x 32768 77 / 75 (not taken
    // there).  Ranges: a workgroup a compute unit, or two where its part is longer than 32 slices; every range costs a partial result that is written and read.  us of
    // product and sum with up to 512 / 256 workgroups, M x N x reduction, bfloat16: 1024 x 1024 x 2500 25.6 / 21.0, 1024 x 1024 x 8192 35.8 / 34.4, 1024 x 2 x 1024 x 8192
    // 51.6 / 56.8; fp32 256 x 256 x 30000 31.5 / 27.1, 1024 x 2 x 256 x 8192 42.5 / 40.7, 300 x 2 x 700 x 30000 116 / 140.
    auto tiles = [&](int64_t bm, int64_t bn) { return (int64_t)cdiv(M, bm) * cdiv(N, bn) * mats; };
    auto ranges = [&](int64_t n) {
        auto upto = [&](int64_t total) { return std::max<int64_t>(1, std::min<int64_t>(slices / 4, total / n)); };
        return slices > 32 * upto(256) ? upto(512) : upto(256);
    };
    int tile = FFT_SMALL;
    const int64_t nw = tiles(256, 256), nm = tiles(128, 128);
    int64_t splits = ranges(tiles(64, 128));
    if (pl == 1 && M > 128 && N > 128 && nw * slices >= 24 * 256) tile = FFT_WIDE, splits = std::max<int64_t>(1, std::min<int64_t>(slices / 4, 256 / nw));
    else if (M > 64 && nm * (slices / 4) >= 192) tile = FFT_MID, splits = ranges(nm);
    const size_t off = ws->off;
    const int rc = launch_tile<true, true, FFK_PARTIAL>(ctx, pl, a, tile, splits, ws, st);
    if (rc) return rc;
    ws->off = off;         // the partial results stay where they are until the next launch
    const int64_t per = cdiv(slices, splits);
    if (per >= slices) return SGNN_OK;
    const int64_t items = M * ((N + 3) / 4) * mats;
    const float *partial = reinterpret_cast<const float *>(ws->base + off);
    const int ranges_ = (int)cdiv(slices, per);
#define SGNN_FFG_REDUCE(ZL_) \
    SGNN_LAUNCH(ctx, st, "ff_reduce_kernel", SGNN_TAG, ff_reduce_kernel<ZL_>, dim3(cdiv(items, 256 / ZL_)), dim3(256), 0, st, partial, ranges_, mats, M, (int)N, C[0], C[mats - 1])
    if (ranges_ >= 32 && items < 256 * 256) SGNN_FFG_REDUCE(16);
    else if (ranges_ >= 8) SGNN_FFG_REDUCE(4);
    else SGNN_FFG_REDUCE(1);
#undef SGNN_FFG_REDUCE
    return SGNN_OK;
}
