// The norms around a block, fused with its gate and residual scale, one kernel each way:
//   b = gamma_post n(z),  w = 1 / (1 + exp(-gate)),  y = alpha x + s w b,  N = gamma_pre n(y),   n(v) = v / sqrt(mean v^2 + eps)
// backward, from the kept y and inverse roots (yh = y ir_pre, zh = z ir_post, D the number of columns):
//   g = dN gamma_pre;  t = dY + ir_pre (g - yh sum(g yh) / D);  dX = alpha t
//   v = t s w;  dgate = t s b w (1 - w) (its row sum where a row has one gate);  h = v gamma_post;  dZ = ir_post (h - zh sum(h zh) / D)
//   ds = sum over the rows of t w b;  dgamma_post of v zh;  dgamma_pre of dN yh
//
// Every matrix is read or written once, which is what bounds these kernels.  A group of G lanes owns a row and keeps it in registers, V values
// (16 bytes) a lane and chunk, CH chunks: G from 8 lanes (eight rows a wavefront: 256 bfloat16 columns would leave half of a whole wavefront idle) to a
// workgroup of 1024 threads.  Row sums are exchanges inside the wavefront, and through LDS between the wavefronts of a row.  Column sums stay in
// registers over all rows of a group, the groups of a workgroup meet in LDS, every workgroup writes one partial sum a column and a second kernel
// adds these in a fixed order: bit-reproducible.  N is taken from y before it is rounded for storage; statistics and sums are fp32.
//
// What else counts is instructions: at 16 fp32 lanes a SIMD some 80 an element are worth its bytes.  The vectors of the columns therefore stay in
// registers over the rows of a group (at most 4096 workgroups, 1024 backward), the parts of a row behind its end are zeros throughout instead of being tested
// for, and a gate costs an exponential and a reciprocal.  2^20 x 256 bfloat16 with a gate for every element: 1552 us with the vectors read and
// the columns tested element by element, 575 here (4.7 TB/s, the rate of a copy 4.8); backward of 32768 x 256 fp32 57 -> 42 (4.8 TB/s).
#include "ff.h"
#include "ff_act.h"

namespace {

template <int G> __device__ __forceinline__ void row_sum(float (&s)[2], float *lds)
{
#pragma unroll
    for (int o = (G < 64 ? G : 64) / 2; o > 0; o >>= 1) {
        s[0] += __shfl_xor(s[0], o, 64);
        s[1] += __shfl_xor(s[1], o, 64);
    }
    if constexpr (G > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();                 // the sums before these have been read
        if ((threadIdx.x & 63) == 0) { lds[2 * wave] = s[0]; lds[2 * wave + 1] = s[1]; }
        __syncthreads();
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int w = 0; w < G / 64; ++w) { s[0] += lds[2 * w]; s[1] += lds[2 * w + 1]; }
    }
}

template <int G> constexpr int threads() { return G > 256 ? G : 256; }

// n fp32 values of a vector at col, `one` where there is no vector, 0 behind its end (so that what is computed there is 0 as well)
template <int V> __device__ __forceinline__ void vector_at(float (&v)[V], const float *p, int col, int left, float one)
{
    if (p) ff_load<FF_T32, V>(v, ff_mat{p, 0, 0}, 0, col, left);
    else
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < left ? one : 0.f;
}

__device__ __forceinline__ float gate_of(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269504088896341f)); }

// the rows' gates: 1 without one; one[] is loaded by every lane of the row
template <int T, int V> __device__ __forceinline__ float row_gate(const ff_norm &a, int64_t row)
{
    if (!a.gate.p || a.gate_cols != 1) return 1.f;
    float one[V];
    ff_load<T, V>(one, a.gate, row, 0, 1);
    return gate_of(one[0]);
}

template <int T, int V, int CH, int G> __global__ __launch_bounds__(threads<G>()) void block_norm_fwd_kernel(ff_norm a)
{
    constexpr int RPW = threads<G>() / G;
    __shared__ float lds[2 * (G > 64 ? G / 64 : 1)];
    const int l = threadIdx.x % G;
    const float inv_d = 1.f / (float)a.d;
    const bool full_gate = a.gate.p && a.gate_cols > 1;
    float post[CH][V], pre[CH][V];            // gamma_post s, gamma_pre
#pragma unroll
    for (int m = 0; m < CH; ++m) {
        const int col = (m * G + l) * V, left = a.d - col;
        float g[V];
        vector_at<V>(g, a.gamma_post, col, left, 1.f);
        vector_at<V>(post[m], a.scale, col, left, 1.f);
        vector_at<V>(pre[m], a.gamma_pre, col, left, 1.f);
#pragma unroll
        for (int i = 0; i < V; ++i) post[m][i] *= g[i];
    }
    // rows are a workgroup's at a time: where a row has several wavefronts they reach every barrier together
    for (int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / G; row < a.rows; row += (int64_t)gridDim.x * RPW) {
        float x[CH][V], z[CH][V], w[CH][V], s[2] = {0.f, 0.f};
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            const int col = (m * G + l) * V, left = a.d - col;
            if (left > 0) {
                if (a.z.p) ff_load<T, V>(z[m], a.z, row, col, left);
                ff_load<T, V>(x[m], a.x, row, col, left);
                if (full_gate) ff_load<T, V>(w[m], a.gate, row, col, left);
            } else
#pragma unroll
                for (int i = 0; i < V; ++i) x[m][i] = z[m][i] = w[m][i] = 0.f;
        }
        if (a.z.p) {
            float ir = row_gate<T, V>(a, row);
            if (a.post) {
#pragma unroll
                for (int m = 0; m < CH; ++m)
#pragma unroll
                    for (int i = 0; i < V; ++i) s[0] = fmaf(z[m][i], z[m][i], s[0]);
                row_sum<G>(s, lds);
                const float r = 1.f / sqrtf(s[0] * inv_d + a.eps);
                if (a.ir_post && l == 0) a.ir_post[row] = r;
                ir *= r;
            }
#pragma unroll
            for (int m = 0; m < CH; ++m)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float b = z[m][i] * ir * post[m][i];
                    if (full_gate) b *= gate_of(w[m][i]);
                    x[m][i] = fmaf(a.alpha, x[m][i], b);
                }
        } else {
#pragma unroll
            for (int m = 0; m < CH; ++m)
#pragma unroll
                for (int i = 0; i < V; ++i) x[m][i] *= a.alpha;
        }
        if (a.y.p) {
#pragma unroll
            for (int m = 0; m < CH; ++m) {
                const int col = (m * G + l) * V, left = a.d - col;
                if (left > 0) ff_store<T, V>(x[m], a.y, row, col, left);
            }
        }
        if (!a.n.p) continue;
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int m = 0; m < CH; ++m)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] = fmaf(x[m][i], x[m][i], s[0]);
        row_sum<G>(s, lds);
        const float ir = 1.f / sqrtf(s[0] * inv_d + a.eps);
        if (a.ir_pre && l == 0) a.ir_pre[row] = ir;
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            const int col = (m * G + l) * V, left = a.d - col;
#pragma unroll
            for (int i = 0; i < V; ++i) x[m][i] *= ir * pre[m][i];
            if (left > 0) ff_store<T, V>(x[m], a.n, row, col, left);
        }
    }
}

template <int T, int V, int CH, int G> __global__ __launch_bounds__(threads<G>()) void block_norm_bwd_kernel(ff_norm a, float *partial)
{
    constexpr int NT = threads<G>(), RPW = NT / G;
    __shared__ float lds[2 * (G > 64 ? G / 64 : 1)];
    __shared__ float red[RPW > 1 ? RPW * G * CH * V : 1];
    const int l = threadIdx.x % G, grp = threadIdx.x / G;
    const float inv_d = 1.f / (float)a.d;
    const bool full_gate = a.gate.p && a.gate_cols > 1;
    float gp[CH][V], sc[CH][V], gn[CH][V];
    float sg[CH][V], ss[CH][V], sp[CH][V];         // sums of v zh, t w zh (times gamma_post at the end), dN yh
#pragma unroll
    for (int m = 0; m < CH; ++m) {
        const int col = (m * G + l) * V, left = a.d - col;
        vector_at<V>(gp[m], a.gamma_post, col, left, 1.f);
        vector_at<V>(sc[m], a.scale, col, left, 1.f);
        vector_at<V>(gn[m], a.gamma_pre, col, left, 1.f);
#pragma unroll
        for (int i = 0; i < V; ++i) ss[m][i] = sp[m][i] = 0.f;
    }
    // rows are a workgroup's at a time, as above
    for (int64_t row = (int64_t)blockIdx.x * RPW + grp; row < a.rows; row += (int64_t)gridDim.x * RPW) {
        float t[CH][V], n[CH][V], y[CH][V], z[CH][V], w[CH][V], s[2] = {0.f, 0.f};
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            const int col = (m * G + l) * V, left = a.d - col;
#pragma unroll
            for (int i = 0; i < V; ++i) t[m][i] = n[m][i] = y[m][i] = z[m][i] = w[m][i] = 0.f;
            if (left <= 0) continue;
            if (a.dn.p) {
                ff_load<T, V>(n[m], a.dn, row, col, left);
                ff_load<T, V>(y[m], a.y, row, col, left);
            }
            if (a.dy.p) ff_load<T, V>(t[m], a.dy, row, col, left);
            if (a.z.p) ff_load<T, V>(z[m], a.z, row, col, left);
            if (full_gate) ff_load<T, V>(w[m], a.gate, row, col, left);
        }
        if (a.dn.p) {
            const float irp = a.in_ir_pre[row];
#pragma unroll
            for (int m = 0; m < CH; ++m)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    y[m][i] *= irp;
                    sp[m][i] = fmaf(n[m][i], y[m][i], sp[m][i]);
                    n[m][i] *= gn[m][i];
                    s[0] = fmaf(n[m][i], y[m][i], s[0]);
                }
            row_sum<G>(s, lds);
            const float mean = s[0] * inv_d;
#pragma unroll
            for (int m = 0; m < CH; ++m)
#pragma unroll
                for (int i = 0; i < V; ++i) t[m][i] = fmaf(irp, fmaf(-y[m][i], mean, n[m][i]), t[m][i]);
        }
        if (a.dx.p) {
#pragma unroll
            for (int m = 0; m < CH; ++m) {
                const int col = (m * G + l) * V, left = a.d - col;
                float dx[V];
#pragma unroll
                for (int i = 0; i < V; ++i) dx[i] = a.alpha * t[m][i];
                if (left > 0) ff_store<T, V>(dx, a.dx, row, col, left);
            }
        }
        if (!a.z.p) continue;
        const float wr = row_gate<T, V>(a, row), irz = a.post ? a.in_ir_post[row] : 1.f;
        // n and y are done with: n becomes h = v gamma_post, y the gate's gradient
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            const int col = (m * G + l) * V, left = a.d - col;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float gate = full_gate ? gate_of(w[m][i]) : wr;
                z[m][i] *= irz;
                const float tg = t[m][i] * gate, g = tg * gp[m][i];
                ss[m][i] = fmaf(tg, z[m][i], ss[m][i]);
                n[m][i] = g * sc[m][i];
                const float hz = n[m][i] * z[m][i];
                s[0] += hz;
                y[m][i] = fmaf(-gate, hz, hz);
                s[1] += y[m][i];
            }
            if (full_gate && a.dgate.p && left > 0) ff_store<T, V>(y[m], a.dgate, row, col, left);
        }
        const bool one_gate = a.dgate.p && a.gate_cols == 1;
        if (a.post || one_gate) row_sum<G>(s, lds);
        if (one_gate && l == 0) {
            float one[V];
#pragma unroll
            for (int i = 0; i < V; ++i) one[i] = s[1];
            ff_store<T, V>(one, a.dgate, row, 0, 1);
        }
        if (a.dz.p) {
            const float mean = a.post ? s[0] * inv_d : 0.f;
#pragma unroll
            for (int m = 0; m < CH; ++m) {
                const int col = (m * G + l) * V, left = a.d - col;
#pragma unroll
                for (int i = 0; i < V; ++i) n[m][i] = irz * fmaf(-z[m][i], mean, n[m][i]);
                if (left > 0) ff_store<T, V>(n[m], a.dz, row, col, left);
            }
        }
    }
    // sums of t w zh: ds is gamma_post times them, dgamma_post s times them
#pragma unroll
    for (int m = 0; m < CH; ++m)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            sg[m][i] = ss[m][i] * sc[m][i];
            ss[m][i] *= gp[m][i];
        }
    if (!partial) return;
    auto out = [&](int q, float (&sum)[CH][V]) {
        float *o = partial + ((int64_t)blockIdx.x * 3 + q) * a.d;
        if constexpr (RPW == 1) {
#pragma unroll
            for (int m = 0; m < CH; ++m)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if ((m * G + l) * V + i < a.d) o[(m * G + l) * V + i] = sum[m][i];
        } else {
            __syncthreads();
#pragma unroll
            for (int m = 0; m < CH; ++m)
#pragma unroll
                for (int i = 0; i < V; ++i) red[grp * (G * CH * V) + (m * G + l) * V + i] = sum[m][i];
            __syncthreads();
            for (int j = threadIdx.x; j < a.d; j += NT) {
                float t = 0.f;
                for (int g = 0; g < RPW; ++g) t += red[g * (G * CH * V) + j];
                o[j] = t;
            }
        }
    };
    out(0, sg);
    out(1, ss);
    out(2, sp);
}

// sum over the workgroups of partial[w][which][col]: 64 interleaved chains a column, sixteen columns a workgroup, and then the chains in order
__global__ __launch_bounds__(1024) void block_norm_sums_kernel(const float *__restrict__ partial, int n, int d, float *__restrict__ o0, float *__restrict__ o1,
                                                               float *__restrict__ o2)
{
    __shared__ float red[1024];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, j = blockIdx.x * 16 + tx;
    float s = 0.f;
    if (j < 3 * d) {
#pragma unroll 8
        for (int w = ty; w < n; w += 64) s += partial[(int64_t)w * 3 * d + j];
    }
    red[threadIdx.x] = s;
    __syncthreads();
    if (ty == 0 && j < 3 * d) {
        float t = 0.f;
#pragma unroll 16
        for (int w = 0; w < 64; ++w) t += red[w * 16 + tx];
        float *o = j < d ? o0 : (j < 2 * d ? o1 : o2);
        if (o) o[j % d] = t;
    }
}

constexpr int MAX_D = 16384, BWD_GROUPS = 1024, FWD_GROUPS = 4096;

// Lanes of a row and chunks of a lane by the row's chunks: the fewest lanes that hold it, one chunk each up to a wavefront.  What is behind a row's end costs as
// much as the rest: 541291 x 64 bfloat16 114 us with 16 lanes a row, 73 with 8, backward 193 and 118; fp32 rows of 129 to 192 chunks by 64 lanes of three instead of
// 256 of one, 150000 x 704 347 and 327, backward 825 and 705, but 5.0 and 6.3 for 400 rows, where a row's own time counts.  (513 to 768 chunks by 256 lanes of
// three are not faster: 30000 x 2536 300 and 306, backward 637 and 697.)
template <int T, int V, class F> int with_shape(int d, int64_t rows, F f)
{
    const int chunks = (d + V - 1) / V;
    if (chunks <= 8) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
    if (chunks <= 16) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 16>());
    if (chunks <= 32) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 32>());
    if (chunks <= 64) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 64>());
    if (chunks <= 128) return f(std::integral_constant<int, 2>(), std::integral_constant<int, 64>());
    if constexpr (V == 4) {
        if (chunks <= 192 && rows >= 2048) return f(std::integral_constant<int, 3>(), std::integral_constant<int, 64>());
    }
    if (chunks <= 256) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 256>());
    if (chunks <= 512) return f(std::integral_constant<int, 2>(), std::integral_constant<int, 256>());
    if (chunks <= 1024) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1024>());
    if constexpr (V == 4) {
        if (chunks > 2048) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 1024>());
    }
    return f(std::integral_constant<int, 2>(), std::integral_constant<int, 1024>());
}

template <int T, int V> int launch_fwd(sgnn_ctx *ctx, const ff_norm &a, hipStream_t st)
{
    return with_shape<T, V>(a.d, a.rows, [&](auto ch, auto g) -> int {
        constexpr int CH = decltype(ch)::value, G = decltype(g)::value, RPW = threads<G>() / G;
        SGNN_LAUNCH(ctx, st, "block_norm_fwd_kernel", SGNN_TAG, (block_norm_fwd_kernel<T, V, CH, G>), dim3((unsigned)std::min<int64_t>(cdiv(a.rows, RPW), FWD_GROUPS)), dim3(threads<G>()), 0, st, a);
        return SGNN_OK;
    });
}

template <int T, int V> int launch_bwd(sgnn_ctx *ctx, const ff_norm &a, ws_alloc *ws, hipStream_t st)
{
    return with_shape<T, V>(a.d, a.rows, [&](auto ch, auto g) -> int {
        constexpr int CH = decltype(ch)::value, G = decltype(g)::value, RPW = threads<G>() / G;
        const bool sums = a.dgamma_post || a.dscale || a.dgamma_pre;
        const unsigned grid = (unsigned)std::min<int64_t>(std::max<int64_t>(cdiv(a.rows, RPW), 1), BWD_GROUPS);
        float *partial = nullptr;
        if (sums) {
            partial = ws->get<float>((size_t)grid * 3 * a.d);
            if (!ws->ok) return sgnn_fail(ctx, SGNN_ERR_CAPACITY, "sgnn_block_norm_bwd: scratch too small: call sgnn_ctx_reserve_ffn");
        }
        SGNN_LAUNCH(ctx, st, "block_norm_bwd_kernel", SGNN_TAG, (block_norm_bwd_kernel<T, V, CH, G>), dim3(grid), dim3(threads<G>()), 0, st, a, partial);
        if (sums)
            SGNN_LAUNCH(ctx, st, "block_norm_sums_kernel", SGNN_TAG, block_norm_sums_kernel, dim3(cdiv(3 * a.d, 16)), dim3(1024), 0, st, partial, (int)grid, a.d,
                        a.dgamma_post, a.dscale, a.dgamma_pre);
        return SGNN_OK;
    });
}

// storage: all of one kind, or mixed
int storage(std::initializer_list<const ff_mat *> ms)
{
    int n16 = 0, n32 = 0;
    for (const ff_mat *m : ms)
        if (m->p) (m->b16 ? n16 : n32)++;
    return n32 == 0 ? FF_T16 : (n16 == 0 ? FF_T32 : FF_TANY);
}

} // namespace

size_t sgnn_block_norm_ws_bytes(uint64_t d) { return (size_t)BWD_GROUPS * 3 * std::min<uint64_t>(d, MAX_D) * 4 + 512; }

int sgnn_launch_block_norm_fwd(sgnn_ctx *ctx, const ff_norm &a, hipStream_t st)
{
    if (a.d > MAX_D) return sgnn_fail(ctx, SGNN_ERR_UNSUPPORTED, "sgnn_block_norm_fwd: rows of %d values are not supported (at most %d)", a.d, MAX_D);
    if (a.rows > 0x7fffffff) return sgnn_fail(ctx, SGNN_ERR_UNSUPPORTED, "sgnn_block_norm_fwd: more than 2^31 - 1 rows");
    if (a.rows == 0) return SGNN_OK;
    const int t = storage({&a.x, &a.z, &a.gate, &a.y, &a.n});
    return t == FF_T16 ? launch_fwd<FF_T16, 8>(ctx, a, st) : (t == FF_T32 ? launch_fwd<FF_T32, 4>(ctx, a, st) : launch_fwd<FF_TANY, 8>(ctx, a, st));
}

int sgnn_launch_block_norm_bwd(sgnn_ctx *ctx, const ff_norm &a, ws_alloc *ws, hipStream_t st)
{
    if (a.d > MAX_D) return sgnn_fail(ctx, SGNN_ERR_UNSUPPORTED, "sgnn_block_norm_bwd: rows of %d values are not supported (at most %d)", a.d, MAX_D);
    if (a.rows > 0x7fffffff) return sgnn_fail(ctx, SGNN_ERR_UNSUPPORTED, "sgnn_block_norm_bwd: more than 2^31 - 1 rows");
    const int t = storage({&a.z, &a.gate, &a.y, &a.dy, &a.dn, &a.dx, &a.dz, &a.dgate});
    return t == FF_T16 ? launch_bwd<FF_T16, 8>(ctx, a, ws, st) : (t == FF_T32 ? launch_bwd<FF_T32, 4>(ctx, a, ws, st) : launch_bwd<FF_TANY, 8>(ctx, a, ws, st));
}
