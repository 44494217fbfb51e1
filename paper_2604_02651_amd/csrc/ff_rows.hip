// Products of a few rows (a trained block that answers for single vertices) with a weight matrix of any size: linear, gated and nt, as in ff_gemm.hip.
//
// A few rows read every weight once for two flop a row: what bounds them is how many weights are on their way at a time.  So the weights go from memory
// straight into operand registers, no LDS and no barrier before the last sum: a wavefront takes pieces of KS reduction steps by CB columns, the up to
// sixteen wavefronts of a workgroup take the pieces of a column strip in turn, and their sums meet in LDS.  Where the
// strips are fewer than the chip's compute units the reduction is split over several workgroups as well: each leaves its sums in scratch, and
// the last one to arrive adds them up in the order of the ranges (bit-reproducible) and applies the epilogue.  No second launch.
//   bfloat16: v_mfma_f32_16x16x32_bf16, fp32: v_mfma_f32_16x16x4_f32 (exact products).  KS = 32 / 16, a lane holds KL = 8 / 4 steps of a row of X and of
//   V columns.  Weights [K x N]: a lane loads V adjacent columns of its KL rows, and pairs of rows are interleaved into operands (fp32 needs none);
//   column tile c of the strip is its columns V i + c.  Weights [N x K] (nt): a lane loads the KL steps of column 16 c + i at once.
#include "ff.h"
#include "ff_act.h"

namespace {

typedef uint32_t u32x2_any2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_any2 __attribute__((aligned(2)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));

enum { FFR_BF16 = 0, FFR_W32 = 1, FFR_F32 = 2 };      // products in bfloat16 of weights stored as bfloat16 / fp32, in fp32

struct ffr_args {
    int M, N;
    int64_t K;                        // of a segment
    int segs;
    ff_mat X[2], W[2];                // of each segment, or projection
    ff_epilogue e;
    uint32_t strips, splits, groups;  // groups: of ROWS rows
    int steps, per_split;             // pieces along the whole reduction, and of one range
    float *partial;                   // [strips][splits][MATS][16 RT][CB]
    uint32_t *arrived;                // [strips], zero between calls
};

// wavefronts of a workgroup: as many as may leave their sums in LDS, at most sixteen
template <int V, int RT, int MATS> constexpr int rows_waves() { return std::min(16, 128 * 1024 / (MATS * 16 * RT * 16 * V * 4)); }

template <int KIND, bool NN, int V, int RT, int MATS> __global__ __launch_bounds__((64 * rows_waves<V, RT, MATS>())) void ff_rows_kernel(ffr_args a)
{
    constexpr int NW = rows_waves<V, RT, MATS>(), KS = KIND == FFR_F32 ? 16 : 32, KL = KS / 4, CB = 16 * V, ROWS = 16 * RT, ES = KIND == FFR_BF16 ? 2 : 4;
    constexpr int WD = NN ? KL * V * ES / 4 : V * KL * ES / 4;             // registers of a piece's weights
    __shared__ float red[MATS][NW][ROWS][CB];
    __shared__ uint32_t last;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, kg = lane >> 4;
    // each XCD has a run of the work, the row groups of a piece of the weights after each other
    const uint32_t total = a.strips * a.splits * a.groups, run = (total + 7) / 8, id = (blockIdx.x & 7) * run + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= run || id >= total) return;
    const uint32_t rest = a.groups > 1 ? id / a.groups : id, group = id - rest * a.groups;
    const uint32_t strip = a.splits > 1 ? rest / a.splits : rest, split = rest - strip * a.splits;
    const int row0 = (int)group * ROWS, n0 = (int)strip * CB;
    const int s_end = min(a.steps, (int)(split + 1) * a.per_split), seg_steps = (int)((a.K + KS - 1) / KS);

    struct piece { uint32_t x[RT][KL * (KIND == FFR_F32 ? 4 : 2) / 4], w[MATS][WD]; };
    auto fetch = [&](piece &p, int s) {
        const int seg = s >= seg_steps ? 1 : 0;
        const int64_t k0 = (int64_t)(s - seg * seg_steps) * KS + KL * kg;
        const int left = (int)min(a.K - k0, (int64_t)KL);             // steps of the lane's KL that exist
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int row = min(row0 + 16 * t + i, a.M - 1);
            if constexpr (KIND != FFR_F32) {
                if (a.X[0].b16 && left >= KL) {
                    const u32x4 d = *reinterpret_cast<const u32x4_any2 *>(static_cast<const u16 *>(a.X[seg].p) + row * a.X[seg].ld + k0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) p.x[t][e] = d[e];
                    continue;
                }
            }
            float v[KL];
            if (left > 0) {
                if constexpr (KIND == FFR_F32) ff_load<FF_T32, KL>(v, a.X[seg], row, k0, left);
                else ff_load<FF_TANY, KL>(v, a.X[seg], row, k0, left);
            } else
#pragma unroll
                for (int e = 0; e < KL; ++e) v[e] = 0.f;
            if constexpr (KIND == FFR_F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) p.x[t][e] = __builtin_bit_cast(uint32_t, v[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) p.x[t][e] = pack_bf16(v[2 * e], v[2 * e + 1]);
            }
        }
#pragma unroll
        for (int q = 0; q < MATS; ++q) {
            const ff_mat &W = a.W[MATS > 1 ? q : seg];
            const unsigned char *base = static_cast<const unsigned char *>(W.p);
            if constexpr (NN) {
                const int col = n0 + V * i;
                const bool whole = col + V <= a.N;
#pragma unroll
                for (int t = 0; t < KL; ++t) {
                    const unsigned char *at = base + (min(k0 + t, a.K - 1) * W.ld + col) * ES;
                    uint32_t *to = p.w[q] + t * (V * ES / 4);
                    if (whole) {
                        if constexpr (V * ES == 16) { const u32x4 d = *reinterpret_cast<const u32x4_any2 *>(at); to[0] = d[0]; to[1] = d[1]; to[2] = d[2]; to[3] = d[3]; }
                        else if constexpr (V * ES == 8) { const u32x2 d = *reinterpret_cast<const u32x2_any2 *>(at); to[0] = d[0]; to[1] = d[1]; }
                        else to[0] = *reinterpret_cast<const u32_any2 *>(at);
                    } else {
#pragma unroll
                        for (int e = 0; e < V * ES / 4; ++e) to[e] = 0;
#pragma unroll
                        for (int c = 0; c < V; ++c)
                            if (col + c < a.N) {
                                if constexpr (ES == 4) to[c] = reinterpret_cast<const uint32_t *>(at)[c];
                                else to[c / 2] |= (uint32_t)reinterpret_cast<const u16 *>(at)[c] << (16 * (c & 1));
                            }
                    }
                    if (t >= left)
#pragma unroll
                        for (int e = 0; e < V * ES / 4; ++e) to[e] = 0;
                }
            } else {
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    const int row = min(n0 + 16 * c + i, a.N - 1);
                    uint32_t *to = p.w[q] + c * (KL * ES / 4);
                    const unsigned char *at = base + (row * W.ld + k0) * ES;
                    if (left >= KL) {
#pragma unroll
                        for (int h = 0; h < KL * ES / 16; ++h) {
                            const u32x4 d = *reinterpret_cast<const u32x4_any2 *>(at + 16 * h);
#pragma unroll
                            for (int e = 0; e < 4; ++e) to[4 * h + e] = d[e];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < KL * ES / 4; ++e) to[e] = 0;
#pragma unroll
                        for (int t = 0; t < KL; ++t)
                            if (t < left) {
                                if constexpr (ES == 4) to[t] = reinterpret_cast<const uint32_t *>(at)[t];
                                else to[t / 2] |= (uint32_t)reinterpret_cast<const u16 *>(at)[t] << (16 * (t & 1));
                            }
                    }
                }
            }
        }
    };
    f32x4 acc[MATS][RT][V];
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int c = 0; c < V; ++c) acc[q][t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const piece &p) {
#pragma unroll
        for (int q = 0; q < MATS; ++q)
#pragma unroll
            for (int c = 0; c < V; ++c) {
                if constexpr (KIND == FFR_F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float b = __builtin_bit_cast(float, NN ? p.w[q][e * V + c] : p.w[q][c * 4 + e]);
#pragma unroll
                        for (int t = 0; t < RT; ++t)
                            acc[q][t][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, p.x[t][e]), b, acc[q][t][c], 0, 0, 0);
                    }
                } else {
                    uint4 b;
                    uint32_t *bp = &b.x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (KIND == FFR_W32) {
                            const uint32_t lo = NN ? p.w[q][2 * e * V + c] : p.w[q][c * 8 + 2 * e], hi = NN ? p.w[q][(2 * e + 1) * V + c] : p.w[q][c * 8 + 2 * e + 1];
                            bp[e] = pack_bf16(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
                        } else if constexpr (NN) {
                            const uint32_t lo = p.w[q][2 * e * (V / 2) + c / 2], hi = p.w[q][(2 * e + 1) * (V / 2) + c / 2];
                            bp[e] = c & 1 ? (lo >> 16) | (hi & 0xffff0000u) : (lo & 0xffffu) | (hi << 16);
                        } else bp[e] = p.w[q][c * 4 + e];
                    }
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        acc[q][t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(p.x[t][0], p.x[t][1], p.x[t][2], p.x[t][3])),
                                                                              __builtin_bit_cast(bf16x8, b), acc[q][t][c], 0, 0, 0);
                }
            }
    };
    {
        // the next piece is on its way while one is multiplied
        int s = (int)split * a.per_split + wave;
        piece p0, p1;
        if (s < s_end) fetch(p0, s);
        for (; s < s_end; s += 2 * NW) {
            if (s + NW < s_end) fetch(p1, s + NW);
            multiply(p0);
            if (s + NW < s_end) {
                if (s + 2 * NW < s_end) fetch(p0, s + 2 * NW);
                multiply(p1);
            }
        }
    }
    // register r of lane (kg, i): row 4 kg + r, column i of a tile
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int c = 0; c < V; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) red[q][wave][16 * t + 4 * kg + r][NN ? V * i + c : 16 * c + i] = acc[q][t][c][r];
    __syncthreads();
    const int rows = min(a.M - row0, ROWS);
    const uint32_t tile = group * a.strips + strip;
    if (a.splits > 1) {
        float *to = a.partial + (size_t)(tile * a.splits + split) * (MATS * ROWS * CB);
        for (int j = threadIdx.x; j < MATS * rows * CB; j += 64 * NW) {
            const int q = j / (rows * CB), r = j / CB % rows, c = j % CB;
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) t += red[q][w][r][c];
            // past the XCD's own L2, so that no cache has to be written back before the count (with a fence for the whole device instead 24 x 4096 x 1024 took
            // 47 us, 9 here)
            __hip_atomic_store(to + (q * ROWS + r) * CB + c, t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0): this wavefront's sums are where every XCD sees them
        __syncthreads();
        if (threadIdx.x == 0) {
            last = __hip_atomic_fetch_add(a.arrived + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (last == a.splits - 1) __hip_atomic_store(a.arrived + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (last != a.splits - 1) return;
    }
    const ff_epilogue &ep = a.e;
    for (int j = threadIdx.x; j < rows * CB; j += 64 * NW) {
        const int r = j / CB, c = j % CB, col = n0 + c;
        const int64_t row = row0 + r;
        if (col >= a.N) continue;
        float v[MATS];
#pragma unroll
        for (int q = 0; q < MATS; ++q) {
            v[q] = 0.f;
            if (a.splits > 1) {
                const float *p = a.partial + (size_t)tile * a.splits * (MATS * ROWS * CB) + (q * ROWS + r) * CB + c;
#pragma unroll 8
                for (uint32_t z = 0; z < a.splits; ++z) v[q] += __hip_atomic_load(p + (size_t)z * (MATS * ROWS * CB), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            } else
#pragma unroll
                for (int w = 0; w < NW; ++w) v[q] += red[q][w][r][c];
            if (ep.bias[q]) v[q] += ep.bias[q][col];
            if (ep.Z[q].p) {
                const float one[4] = {v[q], 0.f, 0.f, 0.f};
                ff_store<FF_TANY, 4>(one, ep.Z[q], row, col, 1);
            }
        }
        float y = 0.f;
        ff_with_act(ep.act, [&](auto act) { y = ff_act<decltype(act)::value>(v[0]); });
        if (MATS > 1) y *= v[MATS - 1];
        else if (ep.R.p) {
            float one[4];
            ff_load<FF_TANY, 4>(one, ep.R, row, col, 1);
            y += one[0];
        }
        const float one[4] = {y, 0.f, 0.f, 0.f};
        ff_store<FF_TANY, 4>(one, ep.Y, row, col, 1);
    }
}

template <int KIND, bool NN, int V, int RT, int MATS> int launch(sgnn_ctx *ctx, ffr_args a, ws_alloc *ws, hipStream_t st)
{
    constexpr int KS = KIND == FFR_F32 ? 16 : 32, CB = 16 * V, NW = rows_waves<V, RT, MATS>(), ROWS = 16 * RT;
    a.strips = cdiv(a.N, CB);
    a.steps = a.segs * (int)cdiv(a.K, KS);
    a.groups = cdiv(a.M, ROWS);
    const uint32_t tiles = a.strips * a.groups;
    // Ranges of the reduction: up to a workgroup a compute unit (of which two at a time find no room where there are more rows), each wavefront with a piece of its
    // own, and at most 16 sums to join.  bfloat16, us with up to 512 workgroups and two pieces a wavefront / here: 24 x 4096 x 1024 8.6 / 7.6, 24 x 4096 x 4096 16.4 / 12.5,
    // 32 x 2048 x 5632 14.8 / 10.4, 1 x 8192 x 8192 28.9 / 26.0 (5.2 TB/s); fp32 24 x 5632 x 1024 16.1 / 11.8, 1 x 8192 x 256 7.9 with 16 ranges, 9.0 with 32.  Two
    // ranges do not pay their join: 1 x 1024 x 4096 5.7 in one, 6.4 in two.
    a.splits = (uint32_t)std::max<int64_t>(1, std::min<int64_t>({256 / (int64_t)tiles, a.steps / NW, 16}));
    if (a.splits == 2 && a.steps < 3 * NW) a.splits = 1;
    a.per_split = (int)cdiv(a.steps, a.splits);
    a.splits = cdiv(a.steps, a.per_split);
    const size_t off = ws->off;
    if (a.splits > 1) {
        a.partial = ws->get<float>((size_t)tiles * a.splits * MATS * ROWS * CB);
        a.arrived = sgnn_ff_arrived(ctx);
        if (!ws->ok) return sgnn_fail(ctx, SGNN_ERR_CAPACITY, "feed-forward operator: scratch too small: call sgnn_ctx_reserve_ffn");
        const int rc = sgnn_ff_open(ctx, st);
        if (rc) return rc;
    }
    char tag[56] = "";
    if (ctx->prof_on) snprintf(tag, sizeof(tag), "%s%s %dx%dx%lld /%u", NN ? "NN" : "NT", MATS > 1 ? " gated" : "", a.M, a.N, (long long)a.K, a.splits);
    auto run = [&]() -> int {
        SGNN_LAUNCH(ctx, st, "ff_rows_kernel", tag, (ff_rows_kernel<KIND, NN, V, RT, MATS>), dim3((tiles * a.splits + 7) / 8 * 8), dim3(64 * NW), 0, st, a);
        return SGNN_OK;
    };
    int rc = run();
    if (a.splits > 1) rc = sgnn_ff_close(ctx, rc, st);
    ws->off = off;         // what the caller launches next on this stream may have the scratch
    return rc;
}

template <int KIND, bool NN, int V, int MATS> int launch_m(sgnn_ctx *ctx, const ffr_args &a, ws_alloc *ws, hipStream_t st)
{
    if (a.M <= 16) return launch<KIND, NN, V, 1, MATS>(ctx, a, ws, st);
    if (a.M <= 32 || MATS > 1) return launch<KIND, NN, V, 2, MATS>(ctx, a, ws, st);
    return launch<KIND, NN, V, 4, MATS>(ctx, a, ws, st);
}

template <bool NN, int MATS> int launch_kind(sgnn_ctx *ctx, const ffr_args &a, bool b16, ws_alloc *ws, hipStream_t st)
{
    // strips of 64 columns (128 bytes of a bfloat16 row), 32 where those are fewer than the compute units
    const bool wide = cdiv(a.N, 64) >= 256;
    if (!b16) return wide ? launch_m<FFR_F32, NN, 4, MATS>(ctx, a, ws, st) : launch_m<FFR_F32, NN, 2, MATS>(ctx, a, ws, st);
    if (a.W[0].b16) return wide ? launch_m<FFR_BF16, NN, 4, MATS>(ctx, a, ws, st) : launch_m<FFR_BF16, NN, 2, MATS>(ctx, a, ws, st);
    return wide ? launch_m<FFR_W32, NN, 4, MATS>(ctx, a, ws, st) : launch_m<FFR_W32, NN, 2, MATS>(ctx, a, ws, st);
}

} // namespace

// Which calls these kernels have: the fewest rows always (each weight is read once), more of them while the products are few, since every 64 rows (32
// gated) read the weights again.  us here / tile kernels, M x K x N, bfloat16: 2048 x 256 x 256 6.2 / 7.7, 512 x 1024 x 1024 9.3 / 14.6, 1024 x 1024 x 1024 16.1 / 15.9,
// 2048 x 1024 x 1024 30 / 15, 512 x 512 x 2048 12.5 / 14.4, 1024 x 512 x 2048 22 / 10, 64 x 4096 x 4096 16.8 / 17.4, 64 x 4096 x 11008 44 / 25; fp32 (whose tile kernels take
// parts that are made first): 512 x 1024 x 1024 21 / 29, 1024 x 1024 x 1024 40 / 32, 64 x 4096 x 4096 39 / 60, 64 x 4096 x 11008 125 / 155, 100 x 4096 x 4096 64 / 65; gated
// 512 x 1024 x 2 x 1024 15.7 / 15.8, fp32 37 / 35.
bool sgnn_ff_rows_take(bool b16, int64_t M, int64_t N, int64_t K, int mats)
{
    return M <= (b16 ? 32 : 64) || (M <= 2048 && (double)M * (double)N * (double)K * mats <= 8e8);
}

size_t sgnn_ff_rows_ws_bytes() { return (size_t)256 * 2 * 64 * 64 * 4 + 256; }

int sgnn_launch_ff_rows(sgnn_ctx *ctx, int64_t M, int64_t N, int64_t K, int segs, int mats, bool nn, bool b16, const ff_mat *X, const ff_mat *W, const ff_epilogue &e,
                        ws_alloc *ws, hipStream_t st)
{
    ffr_args a = {};
    a.M = (int)M; a.N = (int)N; a.K = K; a.segs = segs;
    for (int q = 0; q < 2; ++q) {
        a.X[q] = X[q < segs ? q : 0];
        a.W[q] = W[q < segs * mats ? q : 0];
    }
    a.e = e;
    if (a.W[0].b16 != a.W[1].b16) return SGNN_ERR_UNSUPPORTED;         // the caller's tile kernels read copies of one kind
    if (!nn) return launch_kind<false, 1>(ctx, a, b16, ws, st);
    return mats == 2 ? launch_kind<true, 2>(ctx, a, b16, ws, st) : launch_kind<true, 1>(ctx, a, b16, ws, st);
}
