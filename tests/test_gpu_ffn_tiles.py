"""The feed-forward products at sizes that take every tile: many rows, long reductions, ragged edges.  The 64-bit formulas (ffn_ref.py, with its bounds) are
evaluated for some rows of each result only."""
import numpy as np
import pytest
import torch

import ffn_ref as ref
import paper_2604_02651_amd as sg
from gpu_util import DEV
from test_gpu_ffn import ACT, BF16, F32, TYPES, check, flags, operand_values, vec

pytestmark = pytest.mark.gpu

# M, K, N: more than 2048 rows, or many multiplications (others are the kernels' for few rows)
SHAPES = [(2049, 33, 47), (2100, 2000, 100), (2500, 1000, 130), (2304, 1000, 1000), (4097, 100, 172), (1500, 1100, 600), (8200, 520, 1030), (16400, 64, 1030), (9000, 2056, 513),
          (30011, 200, 531), (70, 4104, 3000)]
_ctx = None


def ctx():
    global _ctx
    if _ctx is None:
        _ctx = sg.Context(0)
        _ctx.reserve_ffn(50000, 1100, 1100)
        _ctx.reserve_ffn(9000, 4200, 3000)
    return _ctx


def normal(shape, dtype, scale=1.0, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, device=DEV, generator=g) * scale).to(dtype)


def host(t):
    return t.double().cpu().numpy()


def some(n, count=150):
    """First, last and some in between"""
    r = np.random.default_rng(n)
    return np.unique(np.concatenate([[0, n - 1, n // 2], r.integers(0, n, min(n, count))]))


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, t):
    M, K, N = shape
    tx, tw, ty, tz = TYPES[t]
    a = ref.ACTS[(M + len(t)) % 5]
    print(shape, t, a, flush=True)
    X, W, Wu, R = normal((M, K), tx, 1.0, 1), normal((K, N), tw, K ** -0.5, 2), normal((K, N), tw, K ** -0.5, 3), normal((M, N), ty, 1.0, 4)
    X[M // 2] *= 2.0 ** -40 if t == "fp32" else 1.0           # a row of another magnitude
    b = normal((N,), F32, 0.3, 5)
    Y, Z, H, G, U = (torch.full((M, N), 77.0, dtype=d, device=DEV) for d in (ty, tz, ty, tz, tz))
    rows = some(M)
    x, w, wu, bb = operand_values(t, host(X[rows])), operand_values(t, host(W)), operand_values(t, host(Wu)), host(b)
    sg.sgnn_linear_fwd(ctx(), X, W, b, ACT[a], flags(t), Y, R=R, Z=Z)
    y, z = ref.linear_fwd(x, w, bb, a, host(R[rows]))
    check(Z[rows], z, "Z"), check(Y[rows], y, "Y")
    again = torch.empty_like(Y)
    sg.sgnn_linear_fwd(ctx(), X, W, b, ACT[a], flags(t), again, R=R)
    assert torch.equal(again, Y)
    sg.sgnn_glu_fwd(ctx(), X, W, Wu, b, None, ACT[a], flags(t), H, G=G, U=U)
    h, g, u = ref.glu_fwd(x, w, wu, bb, None, a)
    check(G[rows], g, "G"), check(U[rows], u, "U"), check(H[rows], h, "H")


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES + [(50000, 512, 1030)], ids=str)
def test_backward(shape, t):
    M, K, N = shape
    tx, tw, ty, tz = TYPES[t]
    a = ref.ACTS[(M + len(t) + 1) % 5]
    print(shape, t, a, flush=True)
    X, W, Wu = normal((M, K), tx, 1.0, 1), normal((K, N), tw, K ** -0.5, 2), normal((K, N), tw, K ** -0.5, 3)
    G, U, dY = normal((M, N), tz, 1.5, 4), normal((M, N), tz, 1.0, 5), normal((M, N), tx, 0.01, 6)
    dY[M // 3] = 0
    X[M // 3] = 3e30                   # a row that adds nothing, whatever its features hold
    dX, dW, dWu = (torch.full(s, 77.0, dtype=ty, device=DEV) for s in ((M, K), (K, N), (K, N)))
    db, du = (torch.full((N,), 77.0, device=DEV) for _ in range(2))
    rows, cols = some(M, 60), some(K, 30)
    w, wu, b16 = operand_values(t, host(W)), operand_values(t, host(Wu)), t != "fp32"
    x = operand_values(t, host(X[:, cols]))

    def verify(Ws, back, outs):
        (dx, _, _) = back(rows)
        check(dX[rows], dx, "dX")
        (_, dws, dbs) = back(slice(None))
        for i, (o, v) in enumerate(outs):
            check(o[cols], dws[i], "dW%d" % i), check(v, dbs[i], "db%d" % i)

    sg.sgnn_linear_bwd(ctx(), X, W, G, ACT[a], flags(t), dY, dX, dW, db)
    g, u, d = host(G), host(U), host(dY)

    def linear(r):
        # all of the rows: a few columns of X are enough for the weights (and W's rows then do not matter)
        return ref.linear_bwd(np.zeros((len(rows), 1)) if r is rows else x, w if r is rows else np.zeros((len(cols), N)), g[r], a, d[r], b16)
    verify([w], linear, [(dW, db)])
    again = torch.empty_like(dX)
    sg.sgnn_linear_bwd(ctx(), X, W, G, ACT[a], flags(t), dY, again, None, None)
    assert torch.equal(again, dX) or b16         # (bfloat16: both products together take another kernel than one)
    check(again[rows], linear(rows)[0], "dX alone")
    alone = torch.empty_like(dW)
    sg.sgnn_linear_bwd(ctx(), X, W, G, ACT[a], flags(t), dY, None, alone, None)
    check(alone[cols], linear(slice(None))[1][0], "dW alone")
    if a == "none":
        a = "silu"
    sg.sgnn_glu_bwd(ctx(), X, W, Wu, G, U, ACT[a], flags(t), dY, dX, dW, dWu, dbg=db, dbu=du)

    def gated(r):
        return ref.glu_bwd(np.zeros((len(rows), 1)) if r is rows else x, *((w, wu) if r is rows else (np.zeros((len(cols), N)),) * 2), g[r], u[r], a, d[r], b16)
    verify([w, wu], gated, [(dW, db), (dWu, du)])


def padded(m, pad):
    """m with `pad` columns of NaN behind every row"""
    wide = torch.full((m.shape[0], m.shape[1] + pad), float("nan"), dtype=m.dtype, device=DEV)
    wide[:, :m.shape[1]] = m
    return wide[:, :m.shape[1]]


# up to 256 columns of X, no gradients of biases: D and dX in one pass, and on either side of the rule for it
@pytest.mark.parametrize("a", ref.ACTS)
@pytest.mark.parametrize("shape", [(32900, 200, 264), (33001, 65, 1032), (32769, 8, 8), (8200, 256, 72), (8319, 129, 520), (65600, 136, 128), (8191, 256, 64)], ids=str)
def test_backward_without_biases(shape, a):
    M, K, N = shape
    print(shape, a, flush=True)
    kept = F32 if a == "gelu" else BF16
    X, W, Wu = normal((M, K), BF16, 1.0, 1), normal((K, N), kept, K ** -0.5, 2), normal((K, N), kept, K ** -0.5, 3)
    G, U, dY = padded(normal((M, N), BF16, 1.5, 4), 8), padded(normal((M, N), BF16, 1.0, 5), 16), padded(normal((M, N), BF16, 0.01, 6), 24)
    if kept is BF16:
        W, Wu = padded(W, 8), padded(Wu, 8)
    dX = padded(torch.full((M, K), 77.0, dtype=kept, device=DEV), 8)
    dW, dWu = (torch.full((K, N), 77.0, dtype=kept, device=DEV) for _ in range(2))
    rows, cols = some(M, 60), some(K, 20)
    x, w, wu = host(X[:, cols]), operand_values("bf16", host(W)), operand_values("bf16", host(Wu))
    g, u, d = host(G), host(U), host(dY)
    few, all_rows = np.zeros((len(rows), 1)), np.zeros((len(cols), N))

    sg.sgnn_glu_bwd(ctx(), X, W, Wu, G, U, ACT[a], flags("bf16"), dY, dX, dW, dWu)
    check(dX[rows], ref.glu_bwd(few, w, wu, g[rows], u[rows], a, d[rows], True)[0], "dX")
    dws = ref.glu_bwd(x, all_rows, all_rows, g, u, a, d, True)[1]
    check(dW[cols], dws[0], "dWg"), check(dWu[cols], dws[1], "dWu")
    assert torch.isnan(dX.as_strided((M, 8), (K + 8, 1), K)).all()
    for out in ((dX, None, None), (dX, None, dWu)):
        before = dX.clone()
        dX.fill_(77.0)
        sg.sgnn_glu_bwd(ctx(), X, W, Wu, G, U, ACT[a], flags("bf16"), dY, *out)
        assert torch.equal(dX, before)
    check(dWu[cols], dws[1], "dWu alone")

    sg.sgnn_linear_bwd(ctx(), X, W, G, ACT[a], flags("bf16"), dY, dX, dW, None)
    check(dX[rows], ref.linear_bwd(few, w, g[rows], a, d[rows], True)[0], "dX")
    check(dW[cols], ref.linear_bwd(x, all_rows, g, a, d, True)[1][0], "dW")
    assert torch.isnan(dX.as_strided((M, 8), (K + 8, 1), K)).all()


# many rows onto up to 256 columns with the gradient of the bias: both products in one pass, weights and their gradient in either type
@pytest.mark.parametrize("kept", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(8300, 96, 200), (9001, 256, 256), (8193, 72, 24), (12000, 200, 100), (8192, 248, 8)], ids=str)
def test_backward_few_columns(shape, kept):
    M, K, N = shape
    print(shape, kept, flush=True)
    X, W, Z, dY = normal((M, K), BF16, 1.0, 1), padded(normal((K, N), kept, K ** -0.5, 2), 8), normal((M, N), BF16, 1.5, 3), normal((M, N), BF16, 0.01, 4)
    dX, dW, db = torch.full((M, K), 77.0, dtype=BF16, device=DEV), padded(torch.full((K, N), 77.0, dtype=kept, device=DEV), 5), torch.full((N,), 77.0, device=DEV)
    rows, cols = some(M, 60), some(K, 20)
    sg.sgnn_linear_bwd(ctx(), X, W, Z, ACT["silu"], flags("bf16"), dY, dX, dW, db)
    z, d, w = host(Z), host(dY), operand_values("bf16", host(W))
    check(dX[rows], ref.linear_bwd(np.zeros((len(rows), 1)), w, z[rows], "silu", d[rows], True)[0], "dX")
    (_, dw, dbs) = ref.linear_bwd(host(X[:, cols]), np.zeros((len(cols), N)), z, "silu", d, True)
    check(dW[cols], dw[0], "dW"), check(db, dbs[0], "db")
    assert torch.isnan(dW.as_strided((K, 5), (N + 5, 1), N)).all()


# many rows and the narrowest matrices.  fp32: two fp16 parts leave out up to 8 E of a product, more than the bound of so few of them allows for
@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(5000, 1, 5), (4099, 3, 1), (3000, 5, 3), (2050, 2, 130), (3001, 4, 4), (70000, 7, 2)], ids=str)
def test_narrow(shape, t):
    M, K, N = shape
    print(shape, t, flush=True)
    dt = TYPES[t][0]
    X, W, Wu, R = normal((M, K), dt, 1.0, 1), normal((K, N), dt, 1.0, 2), normal((K, N), dt, 1.0, 3), normal((M, N), dt, 1.0, 4)
    b, Y, Z, H = normal((N,), F32, 0.3, 5), *(torch.full((M, N), 77.0, dtype=dt, device=DEV) for _ in range(3))
    x, w, wu, bb, r = host(X), host(W), host(Wu), host(b), host(R)

    def check8(got, want, left_out, what):
        check(got, (want[0], want[1] + 8 * ref.E * left_out), what)
    sg.sgnn_linear_fwd(ctx(), X, W, b, ACT["gelu"], flags(t), Y, R=R, Z=Z)
    y, z = ref.linear_fwd(x, w, bb, "gelu", r)
    p, pu = np.abs(x) @ np.abs(w), np.abs(x) @ np.abs(wu)
    check8(Z, z, p, "Z"), check8(Y, y, ref.SLOPE * p, "Y")
    sg.sgnn_glu_fwd(ctx(), X, W, Wu, b, None, ACT["silu"], flags(t), H)
    h, g, u = ref.glu_fwd(x, w, wu, bb, None, "silu")
    check8(H, h, ref.SLOPE * p * (np.abs(u[0]) + 1e-3) + pu * (np.abs(g[0]) + 1), "H")
    dX, dW, dWu, db = torch.full((M, K), 77.0, dtype=dt, device=DEV), *(torch.full((K, N), 77.0, dtype=dt, device=DEV) for _ in range(2)), torch.full((N,), 77.0, device=DEV)
    sg.sgnn_linear_bwd(ctx(), X, W, Z, ACT["silu"], flags(t), R, dX, dW, db)
    zz = host(Z)
    (dx, dws, dbs) = ref.linear_bwd(x, w, zz, "silu", r, t != "fp32")
    d = ref.SLOPE * np.abs(r)
    check8(dX, dx, d @ np.abs(w).T, "dX"), check8(dW, dws[0], np.abs(x).T @ d, "dW"), check(db, dbs[0], "db")
    sg.sgnn_glu_bwd(ctx(), X, W, Wu, Z, H, ACT["silu"], flags(t), R, dX, dW, dWu, dbg=db)
    hh = host(H)
    (dx, dws, dbs) = ref.glu_bwd(x, w, wu, zz, hh, "silu", r, t != "fp32")
    d0, d1 = ref.SLOPE * np.abs(r * hh), np.abs(r) * (np.abs(zz) + 1)
    check8(dX, dx, d0 @ np.abs(w).T + d1 @ np.abs(wu).T, "dX"), check8(dW, dws[0], np.abs(x).T @ d0, "dWg"), check8(dWu, dws[1], np.abs(x).T @ d1, "dWu"), check(db, dbs[0], "dbg")


@pytest.mark.parametrize("shape", [(2304, 200, 130), (2304, 1000, 1000), (40000, 64, 100)], ids=str)
def test_infinities_and_nan_of_many_rows(shape):
    M, K, N = shape
    X, W, Wu = normal((M, K), F32, 1.0, 1), normal((K, N), F32, K ** -0.5, 2), normal((K, N), F32, K ** -0.5, 3)
    Y, H = torch.empty((M, N), device=DEV), torch.empty((M, N), device=DEV)
    X[5, K // 2], X[70, 0], X[M - 1, K - 1], X[9, 3] = float("nan"), float("inf"), -float("inf"), 3.4e38
    sg.sgnn_linear_fwd(ctx(), X, W, None, ACT["relu"], 0, Y)
    sg.sgnn_glu_fwd(ctx(), X, W, Wu, None, None, ACT["none"], 0, H)
    rows = np.unique(np.concatenate([[5, 9, 70, M - 1], some(M, 40)]))
    x, w, wu = host(X[rows]), host(W), host(Wu)
    with np.errstate(invalid="ignore", over="ignore"):
        z, u = x @ w, x @ wu
        want_y, want_h = np.where(np.isnan(z), z, np.maximum(z, 0)), z * u
    got_y, got_h = host(Y[rows]), host(H[rows])
    odd = np.isin(rows, [5, 70, M - 1])
    assert np.isnan(got_y[rows == 5]).all() and np.isnan(got_h[rows == 5]).all()
    assert np.array_equal(np.isposinf(got_y[odd]), np.isposinf(want_y[odd])) and np.array_equal(np.isnan(got_y[odd]), np.isnan(want_y[odd]))
    assert np.array_equal(np.isinf(got_h[odd]), np.isinf(want_h[odd])) and np.array_equal(np.isnan(got_h[odd]), np.isnan(want_h[odd]))
    plain = ~odd & (rows != 9)
    assert np.isfinite(got_y[plain]).all() and np.isfinite(got_h[plain]).all()
    big = rows == 9
    assert np.abs(got_y[big] - want_y[big]).max() <= (K + 12) * ref.E * (np.abs(x[big]) @ np.abs(w)).max()


def test_captured_passes_of_many_rows_replay():
    """The forms of the products that few rows do not reach, captured twice in one graph and replayed between eager calls."""
    c = sg.Context(0)
    c.reserve_ffn(40000, 256, 256)
    B = flags("bf16")
    X, W, dY, Z, U = normal((33000, 192), BF16, 1.0, 1), normal((192, 200), BF16, 0.07, 2), normal((33000, 200), BF16, 0.1, 3), normal((33000, 200), BF16, 1.0, 4), normal((33000, 200), BF16, 1.0, 5)
    Xf, Wf, Rf = normal((9000, 192), F32, 1.0, 6), normal((192, 200), F32, 0.07, 7), normal((9000, 200), F32, 1.0, 8)
    o = [torch.empty(s, dtype=d, device=DEV) for s, d in (((33000, 192), BF16), ((192, 200), BF16), ((192, 200), BF16), ((33000, 192), BF16), ((192, 200), BF16), ((200,), F32),
                                                          ((9000, 200), F32), ((9000, 200), F32))]

    def run():
        sg.sgnn_glu_bwd(c, X, W, W, Z, U, ACT["silu"], B, dY, o[0], o[1], o[2])
        sg.sgnn_linear_bwd(c, X, W, Z, ACT["gelu"], B, dY, o[3], o[4], o[5])
        sg.sgnn_linear_fwd(c, Xf, Wf, None, ACT["gelu"], 0, o[6], R=Rf, Z=o[7])
    run()
    torch.cuda.synchronize()
    want = [a.clone() for a in o]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
        run()
    for k in range(3):
        for a in o:
            a.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o, want)), k
        sg.sgnn_linear_bwd(c, X, W, Z, ACT["relu"], B, dY, o[3], o[4], o[5])
    c.close()


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_offsets_past_32_bits(t):
    """Matrices of more than 2^32 bytes (fp32: 2^33), looked at near their ends; X is zero but for the last rows, so that these alone make the weights' gradients."""
    M, K, N, last = (1 << 21) + 77, 40, 1032, 900
    dt = TYPES[t][0]
    c = sg.Context(0)
    c.reserve_ffn(M, K, N)
    W, Wu = normal((K, N), dt, K ** -0.5, 2), normal((K, N), dt, K ** -0.5, 3)
    X = torch.zeros((M, K), dtype=dt, device=DEV)
    X[M - last:] = normal((last, K), dt, 1.0, 1)
    X[:50] = normal((50, K), dt, 1.0, 9)
    rows = np.unique(np.concatenate([np.arange(50), M - last + some(last, 60)]))
    x, w, wu = host(X[rows]), host(W), host(Wu)
    H, G, U = (torch.empty((M, N), dtype=dt, device=DEV) for _ in range(3))
    sg.sgnn_glu_fwd(c, X, W, Wu, None, None, ACT["silu"], flags(t), H, G=G, U=U)
    h, g, u = ref.glu_fwd(x, w, wu, None, None, "silu")
    check(G[rows], g, "G"), check(U[rows], u, "U"), check(H[rows], h, "H")
    sg.sgnn_linear_fwd(c, X, W, None, ACT["gelu"], flags(t), H, R=U)
    check(H[rows], ref.linear_fwd(x, w, None, "gelu", host(U[rows]))[0], "Y")
    G[M // 2:] += 0.5
    dY = H.mul_(0.01)
    dX, dW, dWu = torch.empty_like(X), torch.empty_like(W), torch.empty_like(Wu)
    X[:50] = 0
    ends = np.arange(M - last, M)
    gr, ur, dr, xe = host(G[rows]), host(U[rows]), host(dY[rows]), host(X[ends])
    ge, ue, de = host(G[ends]), host(U[ends]), host(dY[ends])
    zero = np.zeros((K, N))
    sg.sgnn_glu_bwd(c, X, W, Wu, G, U, ACT["silu"], flags(t), dY, dX, dW, dWu)
    check(dX[rows], ref.glu_bwd(np.zeros((len(rows), 1)), w, wu, gr, ur, "silu", dr, t != "fp32")[0], "dX")
    dws = ref.glu_bwd(xe, zero, zero, ge, ue, "silu", de, t != "fp32")[1]
    check(dW, dws[0], "dWg"), check(dWu, dws[1], "dWu")
    db = torch.empty(N, device=DEV)
    sg.sgnn_linear_bwd(c, X, W, G, ACT["gelu"], flags(t), dY, dX, dW, db)
    check(dX[rows], ref.linear_bwd(np.zeros((len(rows), 1)), w, gr, "gelu", dr, t != "fp32")[0], "dX")
    check(dW, ref.linear_bwd(xe, zero, ge, "gelu", de, t != "fp32")[1][0], "dW")
    n, ir = torch.empty_like(G), torch.empty(M, device=DEV)
    sg.sgnn_block_norm_fwd(c, U, G, None, None, None, None, 1.0, True, 1e-6, H, n, ir, ir.clone())
    z = host(G[rows])
    y = host(U[rows]) + z / np.sqrt((z * z).mean(1, keepdims=True) + 1e-6)
    want = y / np.sqrt((y * y).mean(1, keepdims=True) + 1e-6)
    # a handful of fp32 operations an element and sums of N squares, halved by the root
    tol = (N / 2 + 20) * ref.E * (np.abs(want) + 1)
    assert np.all(np.abs(host(n[rows]) - want) <= tol + (ref.H * (np.abs(want) + tol) if t != "fp32" else 0))
    c.close()
    torch.cuda.empty_cache()


# fp32 onto few columns: the reduction split into ranges, each with its epilogue
@pytest.mark.parametrize("a", ["none", "gelu", "silu"])
@pytest.mark.parametrize("shape", [(2500, 1000, 27), (2051, 2100, 128), (4099, 769, 4), (8191, 3762, 64), (8193, 900, 65), (15167, 1031, 31), (16400, 800, 100)], ids=str)
def test_long_reductions_onto_few_columns(shape, a):
    M, K, N = shape
    print(shape, a, flush=True)
    X, W, b = padded(normal((M, K), F32, 1.0, 1), 3), padded(normal((K, N), F32, K ** -0.5, 2), 1), normal((N,), F32, 0.3, 5)
    Y, Z = (padded(torch.full((M, N), 77.0, device=DEV), 5) for _ in range(2))
    Y.copy_(normal((M, N), F32, 1.0, 4))
    rows = some(M)
    y, z = ref.linear_fwd(host(X[rows]), host(W), host(b), a, host(Y[rows]))
    sg.sgnn_linear_fwd(ctx(), X, W, b, ACT[a], 0, Y, R=Y, Z=Z)          # the residual in place
    check(Z[rows], z, "Z"), check(Y[rows], y, "Y")
    assert torch.isnan(Y.as_strided((M, 5), (N + 5, 1), N)).all() and torch.isnan(Z.as_strided((M, 5), (N + 5, 1), N)).all()
    sg.sgnn_linear_fwd(ctx(), X, W, None, ACT[a], 0, Y)
    check(Y[rows], ref.linear_fwd(host(X[rows]), host(W), None, a, None)[0], "Y")
    if K >= 1000 and N > 4:
        small = sg.Context(0)
        with pytest.raises(sg.SgnnError) as e:
            sg.sgnn_linear_fwd(small, X, W, None, ACT[a], 0, Y)
        assert e.value.code == -2
        small.close()


# norms of widths on either side of every change of the lanes a row has
@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(3001, 30), (3001, 32), (3001, 33), (3001, 64), (3001, 65), (2048, 513), (2051, 704), (2047, 704), (2500, 768), (2500, 769)], ids=str)
def test_norms_of_many_rows(shape, t):
    M, d = shape
    dt = TYPES[t][0]
    X, Z, gate, dY, dN = (normal((M, d), dt, 1.0, i) for i in range(1, 6))
    gp, sc, gn = (normal((d,), F32, 0.5, i) for i in range(6, 9))
    Y, N, irp, irn = torch.empty_like(X), torch.empty_like(X), torch.empty(M, device=DEV), torch.empty(M, device=DEV)
    sg.sgnn_block_norm_fwd(ctx(), X, Z, gate, gp, sc, gn, 0.5, True, 1e-6, Y, N, irp, irn)
    o = [torch.empty_like(X) for _ in range(3)]
    g = [torch.empty(d, device=DEV) for _ in range(3)]
    sg.sgnn_block_norm_bwd(ctx(), Z, Y, gate, gp, sc, gn, 0.5, True, irp, irn, dY, dN, o[0], o[1], o[2], g[0], g[1], g[2])
    # the formulas in float64 by torch, y as it was stored
    x, z, w = X.double(), Z.double(), torch.sigmoid(gate.double())
    zh = z / torch.sqrt((z * z).mean(1, keepdim=True) + 1e-6)
    y = 0.5 * x + sc.double() * w * gp.double() * zh
    half = ref.H if t == "bf16" else ref.E
    # sums of d squares halved by the root, a dozen operations an element, and the rounding as it is stored
    rel = (d / 2 + 20) * ref.E + half
    assert float(((Y.double() - y).abs() / (y.abs() + (0.5 * x).abs() + 1)).max()) <= rel
    nn = gn.double() * y / torch.sqrt((y * y).mean(1, keepdim=True) + 1e-6)
    assert float(((N.double() - nn).abs() / (nn.abs() + 1)).max()) <= 3 * rel
    ys, ir = Y.double(), irn.double()[:, None]
    yh, q = ys * ir, dN.double() * gn.double()
    t_ = dY.double() + ir * (q - yh * (q * yh).mean(1, keepdim=True))
    big = 1 + t_.abs() + (q * ir).abs()
    assert float(((o[0].double() - 0.5 * t_).abs() / big).max()) <= 3 * rel
    h = t_ * sc.double() * w * gp.double()
    dz = irp.double()[:, None] * (h - zh * (h * zh).mean(1, keepdim=True))
    assert float(((o[1].double() - dz).abs() / (1 + dz.abs() + (irp.double()[:, None] * h.abs() * (1 + zh.abs())))).max()) <= 6 * rel
    dg = h * zh * (1 - w)
    assert float(((o[2].double() - dg).abs() / (1 + dg.abs() + (h * zh).abs())).max()) <= 6 * rel
    # sums over M rows: each term to a few roundings of fp32, the sum itself to M of them
    for got, term in ((g[0], t_ * sc.double() * w * zh), (g[1], t_ * w * gp.double() * zh), (g[2], dN.double() * yh)):
        want, mag = term.sum(0), term.abs().sum(0) + M * 1e-3
        assert float(((got.double() - want).abs() / mag).max()) <= (M + 2 * d + 60) * ref.E
