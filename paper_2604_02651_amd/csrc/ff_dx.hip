// The gradients of the pre-activations and the gradient of the input in one pass, all matrices bfloat16, up to 256 columns of X:
//   D0 = dY * act'(Z0)                                       linear
//   D0 = dY * Z1 * act'(Z0),  D1 = dY * act(Z0)              gated
//   dX = D0 W0^T (+ D1 W1^T)                                 [M x K], W [K x N]
// D is written for the gradients of the weights, which are sums over all rows and take it from memory (ff_gemm.hip); here it goes from the registers that
// it was made in to LDS and into the product, so that it is not read back: 131072 x 256 x 704 gated moves 0.99 GB instead of 1.36.
//
// What counts is bytes (a copy of as many takes 205 us; the products take 45 of the matrix pipe's time, the activations 60 of the vector units').  A workgroup has 128
// rows and all columns of dX, and goes through N in steps of 64 columns, whole 128-byte pieces of a row (in steps of 32 it took 253 us instead of 225):
//   - a thread holds eight values of two rows of each operand in registers, requested a step ahead; it makes D of the next step from them, writes it to memory
//     and to LDS (two buffers), and requests the step after it;
//   - W comes by direct loads, two slices of 256 x 64 ahead (three buffers), out of the XCD's L2 where every workgroup finds it;
//   - eight wavefronts of 64 x 64 results, operands 16 bytes a lane, chunks of a row swizzled as in ff_gemm.hip.  Of the two on a SIMD one multiplies first and one
//     makes D first (268 us together, 260 in turns, at 32 columns);
//   - one barrier a slice of W.  Loads and stores past an edge are made and brought to nothing (the last chunk again, bounds of the buffer), so that every step
//     has as many of them and the waits count exactly.
// 131072 x 256 x 704 gated: 225 us, 4.4 TB/s, where D apart and the product apart take 185 and 127.
#include "ff.h"
#include "ff_act.h"

namespace {

constexpr int FFD_BM = 128, FFD_BN = 256, FFD_BK = 64, FFD_WAVES = 8;
constexpr int FFD_STRIP = 64 + 4;                                    // of a row of a wavefront's results on their way out
constexpr int FFD_A = FFD_BM * FFD_BK * 2, FFD_B = FFD_BN * FFD_BK * 2;      // bytes of one operand's slice

struct ffd_args {
    int64_t M;
    int N, K;                         // N a multiple of 8
    const u16 *dY, *Z0, *Z1;
    int64_t ldy, ldz0, ldz1;
    const u16 *W[2]; int64_t ldw;     // [K x N]
    u16 *D; int64_t ldd;              // or null; D1 from column N on
    ff_mat dX;
};

// 16 bytes a lane from p + off.  By a buffer load: behind a global load to LDS the compiler makes every wait for a register one for everything in flight
__device__ __forceinline__ void load_to_lds(const u16 *p, uint32_t off, unsigned char *to)
{
#ifdef __HIP_DEVICE_COMPILE__          // the host's pass does not know 16 bytes
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<u16 *>(p), 0, 0x7fffffff, 0x00020000), STREAM_LPTR(to), 16, off, 0, 0, 0);
#endif
}

__device__ __forceinline__ void write_row(unsigned char *__restrict__ p, const u32x4 &v) { *reinterpret_cast<u32x4 *>(p) = v; }

__device__ __forceinline__ int ffd_swizzle(int l) { return (l >> 1) & 7; }

template <int MATS, int ACT> __global__ __launch_bounds__(64 * FFD_WAVES, 2) void ff_dx_kernel(ffd_args a)
{
    constexpr int BL = FFD_B / 1024 / FFD_WAVES, ROWS = 2, STORES = ROWS * MATS, LOADS = ROWS * (MATS + 1);
    constexpr int WAIT = BL + STORES + LOADS;                      // as many are behind the direct loads of a slice of W when it is used, or more
    extern __shared__ __attribute__((aligned(16))) unsigned char ffd_smem[];
    unsigned char *const w_smem = ffd_smem + 2 * MATS * FFD_A;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 31, kh = lane >> 5;
    const int wm = wave >> 2, wn = wave & 3;
    const int64_t m0 = (int64_t)blockIdx.x * FFD_BM;
    const int steps = (a.N + FFD_BK - 1) / FFD_BK;

    // W: load j of the wavefront is 1 KB, eight rows
    uint32_t off[BL];
#pragma unroll
    for (int j = 0; j < BL; ++j) off[j] = (uint32_t)min(8 * (wave + FFD_WAVES * j) + (lane >> 3), a.K - 1) * (uint32_t)(2 * a.ldw);
    const int b_chunk = (lane & 7) ^ ffd_swizzle(8 * wave + (lane >> 3));      // 64 rows on the swizzle is the same
    auto issue = [&](int s, int q, int slot) {
        const uint32_t c = 2u * (uint32_t)min(s * FFD_BK + 8 * b_chunk, a.N - 8);      // past the end: the last chunk again, nulled where it is used
#pragma unroll
        for (int j = 0; j < BL; ++j) load_to_lds(a.W[q], off[j] + c, w_smem + slot * FFD_B + 1024 * (wave + FFD_WAVES * j));
    };

    // D: the thread's rows and chunk
    const int row = threadIdx.x >> 3, chunk = threadIdx.x & 7;
    const u16 *y_row[ROWS], *z0_row[ROWS], *z1_row[ROWS];
    uint32_t d_at[ROWS];
    constexpr uint32_t BEYOND = 0x80000000u;                      // outside the buffer: the store is dropped
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = m0 + row + 64 * i, from = min(r, a.M - 1);
        y_row[i] = a.dY + from * a.ldy;
        z0_row[i] = a.Z0 + from * a.ldz0;
        z1_row[i] = MATS > 1 ? a.Z1 + from * a.ldz1 : nullptr;
        d_at[i] = a.D && r < a.M ? (uint32_t)(row + 64 * i) * (uint32_t)(2 * a.ldd) + 16u * chunk : BEYOND;
    }
    const uint32_t a_at = row * (FFD_BK * 2) + (chunk ^ ffd_swizzle(row)) * 16;
    const auto d_buffer = __builtin_amdgcn_make_buffer_rsrc(a.D + (a.D ? m0 * a.ldd : 0), 0, 0x7fffffff, 0x00020000);
    struct values { u32x4 y, z0, z1; };
    auto request = [&](int s, values (&v)[ROWS]) __attribute__((always_inline)) {
        const int c = min(s * FFD_BK + 8 * chunk, a.N - 8);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            v[i].y = *reinterpret_cast<const u32x4 *>(y_row[i] + c);
            v[i].z0 = *reinterpret_cast<const u32x4 *>(z0_row[i] + c);
            if (MATS > 1) v[i].z1 = *reinterpret_cast<const u32x4 *>(z1_row[i] + c);
        }
    };
    auto make = [&](int s, const values (&v)[ROWS]) __attribute__((always_inline)) {
        const bool in = s * FFD_BK + 8 * chunk < a.N;
        const u32x4 none = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            u32x4 d0, d1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const ff_act_pair l = ff_act_both<ACT, true>(ff_lo(v[r].z0[i])), h = ff_act_both<ACT, true>(ff_hi(v[r].z0[i]));
                const float yl = ff_lo(v[r].y[i]), yh = ff_hi(v[r].y[i]);
                if (MATS > 1) {
                    d0[i] = pack_bf16(yl * (ff_lo(v[r].z1[i]) * l.d), yh * (ff_hi(v[r].z1[i]) * h.d));
                    d1[i] = pack_bf16(yl * l.f, yh * h.f);
                } else d0[i] = pack_bf16(yl * l.d, yh * h.d);
            }
            const uint32_t to = in ? d_at[r] + (uint32_t)(2 * FFD_BK * s) : BEYOND;
            __builtin_amdgcn_raw_buffer_store_b128(d0, d_buffer, to, 0, 0);
            if (MATS > 1) __builtin_amdgcn_raw_buffer_store_b128(d1, d_buffer, to + (uint32_t)(2 * a.N), 0, 0);
            unsigned char *at = ffd_smem + (s & 1) * (MATS * FFD_A) + a_at + r * 64 * (FFD_BK * 2);
            write_row(at, in ? d0 : none);
            if (MATS > 1) write_row(at + FFD_A, in ? d1 : none);
        }
    };

    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    const int at_row = li * (FFD_BK * 2) + (kh ^ ffd_swizzle(li)) * 16;
    auto multiply = [&](int s, int q, int slot) __attribute__((always_inline)) {
        const unsigned char *d = ffd_smem + (s & 1) * (MATS * FFD_A) + q * FFD_A + 64 * wm * (FFD_BK * 2), *w = w_smem + slot * FFD_B + 64 * wn * (FFD_BK * 2);
#pragma unroll
        for (int ks = 0; ks < FFD_BK / 16; ++ks) {
            u32x4 fa[2], fb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) fa[i] = read_row(d + 32 * i * (FFD_BK * 2) + (at_row ^ (32 * ks)));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                fb[j] = read_row(w + 32 * j * (FFD_BK * 2) + (at_row ^ (32 * ks)));
                fb[j] &= FFD_BK * s + 16 * ks + 8 * kh < a.N ? 0xffffffffu : 0u;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fb[j]), __builtin_bit_cast(bf16x8, fa[i]), acc[i][j], 0, 0, 0);
        }
    };
    auto next = [](int slot) { return slot == 2 ? 0 : slot + 1; };
    auto meet = [] {
        STREAM_WAIT_VMCNT(WAIT);                                   // the slice of W has landed (this wavefront's part)
        __builtin_amdgcn_s_waitcnt(0xC07F);                        // lgkmcnt(0): its part of D is in LDS
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();                              // everybody's part; and everybody is through the slice before
        asm volatile("" ::: "memory");
    };
    values v[ROWS];
    request(0, v);
    asm volatile("" ::: "memory");
    issue(0, 0, 0);
    asm volatile("" ::: "memory");
    make(0, v);
    asm volatile("" ::: "memory");
    request(1, v);
    asm volatile("" ::: "memory");
    issue(MATS == 2 ? 0 : 1, MATS - 1, 1);
    int slot = 0;                                                  // of the slice of W to be multiplied
    for (int s = 0; s < steps; ++s) {
        meet();
        issue(MATS == 2 ? s + 1 : s + 2, 0, next(next(slot)));
        asm volatile("" ::: "memory");
        // the wavefronts that share a SIMD (0 and 4, ...) take turns: one multiplies, one makes D of the next step
        if (wm) multiply(s, 0, slot);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {          // nothing of D is made before here (the compiler would, and wait for the operands before the barrier)
            asm volatile("" : "+v"(v[i].y), "+v"(v[i].z0) : : "memory");
            if (MATS > 1) asm volatile("" : "+v"(v[i].z1));
        }
        make(s + 1, v);
        asm volatile("" ::: "memory");
        request(s + 2, v);
        asm volatile("" ::: "memory");
        if (!wm) multiply(s, 0, slot);
        slot = next(slot);
        if (MATS == 2) {
            meet();
            issue(s + 1, 1, next(next(slot)));
            asm volatile("" ::: "memory");
            multiply(s, 1, slot);
            slot = next(slot);
        }
    }
    STREAM_WAIT_VMCNT(0);       // the repeated loads past the end are still in flight: nothing may use the LDS before they land
    __syncthreads();

    // register r of lane (kh, li) is row li, column 8 (r / 4) + 4 kh + r % 4 of a block: through a strip of LDS of the wavefront's own, 32 rows at a time, so that
    // a lane has eight adjacent columns
    float *const strip = reinterpret_cast<float *>(ffd_smem) + wave * 32 * FFD_STRIP;
    const int c = 8 * (lane & 7), col = 64 * wn + c;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4 *>(strip + li * FFD_STRIP + 32 * j + 8 * q + 4 * kh) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
#pragma unroll 1
        for (int r0 = 0; r0 < 32; r0 += 8) {
            const int r = r0 + (lane >> 3);
            const int64_t to = m0 + 64 * wm + 32 * i + r;
            if (to >= a.M || col >= a.K) continue;
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(strip + r * FFD_STRIP + c), hi = *reinterpret_cast<const f32x4 *>(strip + r * FFD_STRIP + c + 4);
            const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            ff_store<FF_TANY, 8>(x, a.dX, to, col, a.K - col);
        }
    }
}

template <int MATS, int ACT> int launch_dx(sgnn_ctx *ctx, const ffd_args &a, hipStream_t st)
{
    constexpr int LDS = std::max(2 * MATS * FFD_A + 3 * FFD_B, FFD_WAVES * 32 * FFD_STRIP * 4);
    SGNN_HIP(ctx, (sgnn_allow_lds<&ff_dx_kernel<MATS, ACT>>(ctx, LDS)));
    SGNN_LAUNCH(ctx, st, "ff_dx_kernel", MATS > 1 ? "gated" : "linear", (ff_dx_kernel<MATS, ACT>), dim3(cdiv(a.M, FFD_BM)), dim3(64 * FFD_WAVES), LDS, st, a);
    return SGNN_OK;
}

template <int MATS> int launch_dx_act(sgnn_ctx *ctx, int act, const ffd_args &a, hipStream_t st)
{
    switch (act) {
    case SGNN_ACT_RELU: return launch_dx<MATS, SGNN_ACT_RELU>(ctx, a, st);
    case SGNN_ACT_GELU: return launch_dx<MATS, SGNN_ACT_GELU>(ctx, a, st);
    case SGNN_ACT_GELU_TANH: return launch_dx<MATS, SGNN_ACT_GELU_TANH>(ctx, a, st);
    case SGNN_ACT_SILU: return launch_dx<MATS, SGNN_ACT_SILU>(ctx, a, st);
    default: return launch_dx<MATS, SGNN_ACT_NONE>(ctx, a, st);
    }
}

} // namespace

// Returns SGNN_ERR_UNSUPPORTED without launching anything for what the kernel does not handle.  W chunked, of one leading dimension; D [M x mats N] or null.
int sgnn_launch_ff_dx(sgnn_ctx *ctx, int64_t M, int64_t N, int64_t K, int mats, int act, const ff_mat &dY, const ff_mat *Z, const ff_op *W, const ff_mat &D, const ff_mat &dX,
                      hipStream_t st)
{
    auto readable = [&](const ff_mat &m) { return m.b16 && ff_chunked(m.p, N, m.ld); };
    if (K > FFD_BN || N > (1 << 20) || !readable(dY) || !readable(Z[0]) || (mats > 1 && (!readable(Z[1]) || W[0].ld != W[1].ld)) || M > ((int64_t)1 << 36)) return SGNN_ERR_UNSUPPORTED;
    ffd_args a = {};
    a.M = M; a.N = (int)N; a.K = (int)K;
    a.dY = static_cast<const u16 *>(dY.p); a.ldy = dY.ld;
    a.Z0 = static_cast<const u16 *>(Z[0].p); a.ldz0 = Z[0].ld;
    if (mats > 1) { a.Z1 = static_cast<const u16 *>(Z[1].p); a.ldz1 = Z[1].ld; }
    for (int q = 0; q < mats; ++q) a.W[q] = W[q].p;
    a.ldw = W[0].ld;
    a.D = static_cast<u16 *>(const_cast<void *>(D.p)); a.ldd = D.ld;
    a.dX = dX;
    return mats > 1 ? launch_dx_act<2>(ctx, act, a, st) : launch_dx_act<1>(ctx, act, a, st);
}
