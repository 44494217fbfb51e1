"""The feed-forward operators against their formulas in 64 bits (ffn_ref.py, which also derives how far a result may be off)."""
import numpy as np
import pytest
import torch

import ffn_ref as ref
import paper_2604_02651_amd as sg
from gpu_util import DEV

pytestmark = pytest.mark.gpu

ACT = dict(none=sg.SGNN_ACT_NONE, relu=sg.SGNN_ACT_RELU, gelu=sg.SGNN_ACT_GELU, gelu_tanh=sg.SGNN_ACT_GELU_TANH, silu=sg.SGNN_ACT_SILU)
F32, BF16 = torch.float32, torch.bfloat16
# storage of (inputs X and dY, weights, results, kept pre-activations)
TYPES = {"fp32": (F32, F32, F32, F32), "bf16": (BF16, BF16, BF16, BF16), "mixed": (F32, BF16, F32, BF16), "master": (BF16, F32, BF16, F32)}
SHAPES = [(1, 1, 1), (1, 64, 256), (2, 5, 3), (7, 16, 8), (16, 1000, 130), (17, 33, 257), (64, 64, 64), (130, 72, 200), (129, 531, 47), (257, 200, 531),
          (1000, 256, 704), (4097, 100, 172)]

_ctx = None


def ctx():
    global _ctx
    if _ctx is None:
        _ctx = sg.Context(0)
        _ctx.reserve_ffn(1 << 14, 1100, 1100)
    return _ctx


def flags(t):
    return 0 if t == "fp32" else sg.SGNN_BF16_MFMA


def values(r, shape, dtype, scale=1.0):
    """float64 values that the storage type holds exactly"""
    v = (r.standard_normal(shape) * scale).astype(np.float32)
    return ref.round_bf16(v) if dtype == BF16 else v.astype(np.float64)


def dev(v, dtype, pad=0, off=0):
    """On the GPU with `pad` more columns between rows (holding NaN) and `off` elements in front."""
    if v is None:
        return None
    rows, cols = v.shape
    buf = torch.full((off + rows * (cols + pad) + 8,), float("nan"), dtype=dtype, device=DEV)
    t = buf[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.tensor(v, dtype=torch.float64).to(dtype))
    return t


def vec(v):
    return None if v is None else torch.tensor(v, dtype=F32, device=DEV)


def out(rows, cols, dtype, pad=0, off=0):
    buf = torch.full((off + rows * (cols + pad) + 8,), 77.0, dtype=dtype, device=DEV)
    t = buf[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.around = lambda: torch.cat([buf[:off], buf[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, cols:].reshape(-1), buf[off + rows * (cols + pad):]])
    return t


def check(got, want, what):
    """Every element within its bound, plus the rounding of its storage; nothing around it written."""
    x, e = want
    if got.dtype == BF16:
        e = e + ref.H * (np.abs(x) + e) + 2.0 ** -133
    else:
        e = e + ref.E * np.abs(x) + 2.0 ** -149
    d = np.abs(got.double().cpu().numpy() - x)
    assert d.shape == x.shape and np.all(d <= e), "%s: %g of the bound at %s" % (what, (d / e).max(), np.unravel_index(np.argmax(d / e), d.shape))
    if hasattr(got, "around"):
        assert bool((got.around() == 77.0).all()), what + ": written outside"


def operand_values(t, W):
    """what the products read of weights stored as fp32"""
    return ref.round_bf16(W) if t != "fp32" else W


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_linear_forward(shape, t):
    M, K, N = shape
    tx, tw, ty, tz = TYPES[t]
    r = np.random.default_rng(M + 3 * K + 7 * N)
    for i, a in enumerate(ref.ACTS):
        print(shape, t, a, flush=True)
        pad, off = (0, 0) if i % 2 else (i + 1, i)
        X, W, b, R = values(r, (M, K), tx), values(r, (K, N), tw, K ** -0.5), values(r, (N,), F32, 0.3), values(r, (M, N), ty)
        X[0, 0] = 0.0
        y, z = ref.linear_fwd(operand_values(t, X), operand_values(t, W), b if i != 2 else None, a, R if i != 3 else None)
        Y, Z = out(M, N, ty, pad, off), out(M, N, tz, pad, off)
        sg.sgnn_linear_fwd(ctx(), dev(X, tx, pad, off), dev(W, tw, pad, off), vec(b) if i != 2 else None, ACT[a], flags(t), Y, R=dev(R, ty, pad, off) if i != 3 else None, Z=Z)
        check(Z, z, "Z")
        check(Y, y, "Y")
        Y2 = out(M, N, ty)
        if i != 3:
            Y2.copy_(dev(R, ty))
        sg.sgnn_linear_fwd(ctx(), dev(X, tx), dev(W, tw), vec(b) if i != 2 else None, ACT[a], flags(t), Y2, R=Y2 if i != 3 else None)       # nothing kept, R in place
        check(Y2, y, "Y in place")


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_glu_forward(shape, t):
    M, K, N = shape
    tx, tw, ty, tz = TYPES[t]
    r = np.random.default_rng(M + 5 * K + 11 * N)
    for i, a in enumerate(ref.ACTS[1:]):
        print(shape, t, a, flush=True)
        pad, off = (0, 0) if i % 2 else (i + 1, i)
        X, Wg, Wu = values(r, (M, K), tx), values(r, (K, N), tw, K ** -0.5), values(r, (K, N), tw, K ** -0.5)
        bg, bu = (values(r, (N,), F32, 0.3) for _ in range(2)) if i < 2 else (None, None)
        h, g, u = ref.glu_fwd(operand_values(t, X), operand_values(t, Wg), operand_values(t, Wu), bg, bu, a)
        Y, G, U = out(M, N, ty, pad, off), out(M, N, tz, pad, off), out(M, N, tz, pad, off)
        sg.sgnn_glu_fwd(ctx(), dev(X, tx, pad, off), dev(Wg, tw, pad, off), dev(Wu, tw, 2 * pad, off), vec(bg), vec(bu), ACT[a], flags(t), Y, G=G, U=U)
        check(G, g, "G"), check(U, u, "U"), check(Y, h, "H")
        Y2 = out(M, N, ty)
        sg.sgnn_glu_fwd(ctx(), dev(X, tx), dev(Wg, tw), dev(Wu, tw), vec(bg), vec(bu), ACT[a], flags(t), Y2, U=out(M, N, tz) if i % 2 else None)
        check(Y2, h, "H alone")


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_linear_backward(shape, t):
    M, K, N = shape
    tx, tw, ty, tz = TYPES[t]
    r = np.random.default_rng(M + 13 * K + 17 * N)
    for i, a in enumerate(ref.ACTS):
        print(shape, t, a, flush=True)
        pad, off = (0, 0) if i % 2 else (i + 1, i)
        X, W, Z, dY = values(r, (M, K), tx), values(r, (K, N), tw, K ** -0.5), values(r, (M, N), tz, 1.5), values(r, (M, N), tx, 0.01)
        (dx, dw, db) = ref.linear_bwd(operand_values(t, X), operand_values(t, W), Z, a, dY, t != "fp32")
        args = lambda p, o: (ctx(), dev(X, tx, p, o), dev(W, tw, p, o), dev(Z, tz, p, o) if a != "none" or i % 2 else None, ACT[a], flags(t), dev(dY, tx, p, o))      # noqa: E731
        dX, dW, dB = out(M, K, ty, pad, off), out(K, N, ty, pad, off), torch.full((N,), 77.0, device=DEV)
        sg.sgnn_linear_bwd(*args(pad, off), dX, dW, dB)
        check(dX, dx, "dX"), check(dW, dw[0], "dW"), check(dB, db[0], "dbias")
        again = out(K, N, ty)
        sg.sgnn_linear_bwd(*args(pad, off), None, again, None)
        assert torch.equal(again, dW)
        again = out(M, K, ty)
        sg.sgnn_linear_bwd(*args(0, 0), again, None, None)
        check(again, dx, "dX alone")
        alone = torch.zeros(N, device=DEV)
        sg.sgnn_linear_bwd(*args(0, 0), None, None, alone)
        check(alone, db[0], "dbias alone")


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_glu_backward(shape, t):
    M, K, N = shape
    tx, tw, ty, tz = TYPES[t]
    r = np.random.default_rng(M + 19 * K + 23 * N)
    for i, a in enumerate(ref.ACTS[1:]):
        print(shape, t, a, flush=True)
        pad, off = (0, 0) if i % 2 else (i + 1, i)
        X, Wg, Wu = values(r, (M, K), tx), values(r, (K, N), tw, K ** -0.5), values(r, (K, N), tw, K ** -0.5)
        G, U, dH = values(r, (M, N), tz, 1.5), values(r, (M, N), tz), values(r, (M, N), tx, 0.01)
        dx, dw, db = ref.glu_bwd(operand_values(t, X), operand_values(t, Wg), operand_values(t, Wu), G, U, a, dH, t != "fp32")
        args = lambda p, o: (ctx(), dev(X, tx, p, o), dev(Wg, tw, p, o), dev(Wu, tw, 3 * p, o), dev(G, tz, p, o), dev(U, tz, p, o), ACT[a], flags(t), dev(dH, tx, p, o))   # noqa: E731
        dX, dWg, dWu = out(M, K, ty, pad, off), out(K, N, ty, pad, off), out(K, N, ty, 2 * pad, off)
        bg, bu = (torch.full((N,), 77.0, device=DEV) for _ in range(2))
        sg.sgnn_glu_bwd(*args(pad, off), dX, dWg, dWu, dbg=bg, dbu=bu)
        check(dX, dx, "dX"), check(dWg, dw[0], "dWg"), check(dWu, dw[1], "dWu"), check(bg, db[0], "dbg"), check(bu, db[1], "dbu")
        x2, w2, b2 = out(M, K, ty), out(K, N, ty), torch.zeros(N, device=DEV)
        sg.sgnn_glu_bwd(*args(0, 0), x2, None, w2, dbu=b2)
        check(x2, dx, "dX"), check(w2, dw[1], "dWu alone"), check(b2, db[1], "dbu alone")


# ---- norms ---------------------------------------------------------------------------------------

NORM_SHAPES = [(1, 1), (3, 2), (5, 8), (1, 4096), (9, 47), (100, 128), (257, 256), (33, 260), (70, 500), (31, 512), (20, 1000), (9, 1030), (6, 2049), (3, 4100), (2, 8200),
               (2, 16384), (5000, 64)]


def norm_bound(x, terms, b16_terms=0.0):
    """A result made of few terms, whose largest magnitude is `terms`, by way of a row sum of d squares or products: 2^-18 of that (row sums of up to 16384
    positive fp32 terms in a tree of depth under 40, an inverse root, some ten operations)."""
    return x, 2.0 ** -18 * terms + b16_terms


@pytest.mark.parametrize("t", ["fp32", "bf16", "mixed"])
@pytest.mark.parametrize("shape", NORM_SHAPES, ids=str)
@pytest.mark.parametrize("gate,post,pre", [(None, True, True), ("row", True, True), ("full", True, False), ("full", False, True), ("row", False, False)])
def test_block_norm(shape, gate, post, pre, t):
    M, d = shape
    tx, tz = {"fp32": (F32, F32), "bf16": (BF16, BF16), "mixed": (F32, BF16)}[t]
    r = np.random.default_rng(29 * M + d + post)
    pad, off = (3, 1) if d % 2 else (0, 0)
    X, Z, dY, dN = values(r, (M, d), tx), values(r, (M, d), tz, 1.5), values(r, (M, d), tx, 0.01), values(r, (M, d), tz, 0.01)
    gt = None if gate is None else values(r, (M, 1 if gate == "row" else d), tz, 2.0)
    gp, sc, gn = (1 + 0.3 * values(r, (d,), F32) for _ in range(3))
    gp, sc, gn = (ref.np.asarray(v, np.float32).astype(np.float64) for v in (gp, sc, gn))
    gp = gp if post else None
    gn = gn if pre else None
    eps, alpha = 1e-5, 0.75
    y, n, ip, iq = ref.block_norm_fwd(X, Z, gt, gp, sc, gn, alpha, post, eps)
    Y, N = out(M, d, tx, pad, off), out(M, d, tz, pad, off) if pre else None
    a, b = (torch.zeros(M, device=DEV) for _ in range(2))
    largest = np.abs(alpha * X) + np.abs(y - alpha * X)
    sg.sgnn_block_norm_fwd(ctx(), dev(X, tx, pad, off), dev(Z, tz, pad, off), dev(gt, tz), vec(gp), vec(sc), vec(gn), alpha, post, eps, Y, N, a if post else None, b if pre else None)
    check(Y, norm_bound(y, largest), "Y")
    if post:
        check(a, norm_bound(ip, ip), "ir_post")
    if pre:
        # the mean square of y moves with y's own errors: relative to its row's size
        size = (largest ** 2).mean(1, keepdims=True) ** 0.5
        check(N, norm_bound(n, np.abs(gn) * iq[:, None] * (largest + np.abs(y) * size * iq[:, None])), "N")
        check(b, norm_bound(iq, iq * (1 + size[:, 0] * iq)), "ir_pre")
    # backward from what is kept
    Yk, ipk, iqk = Y.double().cpu().numpy(), a.double().cpu().numpy(), b.double().cpu().numpy()
    o = ref.block_norm_bwd(Z, Yk, ipk, iqk, dY, dN if pre else None, gt, gp, sc, gn, alpha, post)
    got = dict(dX=out(M, d, tx, pad, off), dZ=out(M, d, tz, pad, off), dgate=None if gt is None else out(*gt.shape, tz), dgamma_post=torch.zeros(d, device=DEV) if post else None,
               dscale=torch.zeros(d, device=DEV), dgamma_pre=torch.zeros(d, device=DEV) if pre else None)
    args = (ctx(), dev(Z, tz, pad, off), Y if pre else None, dev(gt, tz), vec(gp), vec(sc), vec(gn), alpha, post, a if post else None, b if pre else None, dev(dY, tx, pad, off),
            dev(dN, tz, pad, off) if pre else None)
    sg.sgnn_block_norm_bwd(*args, got["dX"], got["dZ"], got["dgate"], got["dgamma_post"], got["dscale"], got["dgamma_pre"])
    # magnitudes of the terms of each
    tt = np.abs(dY)
    if pre:
        yh, g = np.abs(Yk) * iqk[:, None], np.abs(dN * gn)
        tt = tt + iqk[:, None] * (g + yh * (g * yh).mean(1, keepdims=True))
    zh = np.abs(Z) * (ipk[:, None] if post else 1)
    bb, w, s = zh * (np.abs(gp) if post else 1), 1 if gt is None else 1 / (1 + np.exp(-gt)), np.abs(sc)
    v = tt * s * w
    check(got["dX"], norm_bound(o["dX"], alpha * tt), "dX")
    if post:
        h = v * np.abs(gp)
        check(got["dZ"], norm_bound(o["dZ"], ipk[:, None] * (h + zh * (h * zh).mean(1, keepdims=True))), "dZ")
        check(got["dgamma_post"], (o["dgamma_post"], ((M + 4) * ref.E + 2.0 ** -18) * (v * zh).sum(0)), "dgamma_post")
    else:
        check(got["dZ"], norm_bound(o["dZ"], v), "dZ")
    check(got["dscale"], (o["dscale"], ((M + 4) * ref.E + 2.0 ** -18) * (tt * w * bb).sum(0)), "dscale")
    if gt is not None:
        terms = tt * s * bb * w
        check(got["dgate"], norm_bound(o["dgate"], terms.sum(1, keepdims=True) if gate == "row" else terms), "dgate")
    if pre:
        check(got["dgamma_pre"], (o["dgamma_pre"], ((M + 4) * ref.E + 2.0 ** -18) * (np.abs(dN) * yh).sum(0)), "dgamma_pre")
    # the same without the sums, in place, and once more with them: bit for bit
    dx, dz = dev(dY, tx, pad, off), dev(dN, tz, pad, off)
    sg.sgnn_block_norm_bwd(*args[:11], dx, dz if pre else None, dx, dz, None, None, None, None)
    assert torch.equal(dx, got["dX"]) and torch.equal(dz, got["dZ"])
    s2 = torch.zeros(d, device=DEV)
    sg.sgnn_block_norm_bwd(*args, None, None, None, None, s2, None)
    assert torch.equal(s2, got["dscale"])


def test_block_norm_in_front_of_the_first_block():
    r = np.random.default_rng(1)
    X, g = values(r, (70, 200), F32), 1 + 0.1 * values(r, (200,), F32)
    g = g.astype(np.float32).astype(np.float64)
    _, n, _, iq = ref.block_norm_fwd(X, None, gamma_pre=g, eps=1e-6)
    N, ir, x = out(70, 200, F32), torch.zeros(70, device=DEV), dev(X, F32)
    sg.sgnn_block_norm_fwd(ctx(), x, None, None, None, None, vec(g), 1.0, False, 1e-6, None, N, None, ir)
    check(N, norm_bound(n, 2 * np.abs(n)), "N")
    dN, dY = values(r, (70, 200), F32), values(r, (70, 200), F32)
    o = ref.block_norm_bwd(None, X, None, ir.double().cpu().numpy(), dY, dN, gamma_pre=g)
    dX, dg = out(70, 200, F32), torch.zeros(200, device=DEV)
    sg.sgnn_block_norm_bwd(ctx(), None, x, None, None, None, vec(g), 1.0, False, None, ir, dev(dY, F32), dev(dN, F32), dX, None, dgamma_pre=dg)
    size = np.abs(dY) + iq[:, None] * np.abs(dN * g) + iq[:, None] ** 2 * np.abs(X) * (np.abs(dN * g) * np.abs(X) * iq[:, None]).mean(1, keepdims=True)
    check(dX, norm_bound(o["dX"], size), "dX")
    check(dg, (o["dgamma_pre"], (74 * ref.E + 2.0 ** -18) * np.abs(dN * X * iq[:, None]).sum(0)), "dgamma_pre")
    sg.sgnn_block_norm_bwd(ctx(), None, x, None, None, None, vec(g), 1.0, False, None, ir, None, dev(dN, F32), dX, None)
    o = ref.block_norm_bwd(None, X, None, ir.double().cpu().numpy(), None, dN, gamma_pre=g)
    check(dX, norm_bound(o["dX"], size), "dX without dY")


# ---- what real calls bring along -------------------------------------------------------------------

@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_batches_without_rows(t):
    tx, tw, ty, tz = TYPES[t]
    X, W, b = torch.empty((0, 24), dtype=tx, device=DEV), torch.ones((24, 40), dtype=tw, device=DEV), torch.ones(40, device=DEV)
    Y = torch.empty((0, 40), dtype=ty, device=DEV)
    sg.sgnn_linear_fwd(ctx(), X, W, b, ACT["gelu"], flags(t), Y, Z=torch.empty_like(Y))
    sg.sgnn_glu_fwd(ctx(), X, W, W, b, b, ACT["silu"], flags(t), Y)
    dW, dU, db, du = out(24, 40, ty, 3, 1), out(24, 40, ty), torch.ones(40, device=DEV), torch.ones(40, device=DEV)
    sg.sgnn_linear_bwd(ctx(), X, W, Y, ACT["gelu"], flags(t), Y, torch.empty_like(X), dW, db)
    check(dW, (np.zeros((24, 40)), np.zeros((24, 40))), "dW")
    assert not db.any()
    dW.fill_(1), db.fill_(1)
    sg.sgnn_glu_bwd(ctx(), X, W, W, Y, Y, ACT["gelu"], flags(t), Y, torch.empty_like(X), dW, dU, dbg=db, dbu=du)
    assert not dW.any() and not dU.any() and not db.any() and not du.any()
    g = torch.ones(24, device=DEV)
    sg.sgnn_block_norm_fwd(ctx(), X, X, None, None, None, None, 1.0, True, 1e-6, X, torch.empty_like(X))
    sg.sgnn_block_norm_bwd(ctx(), X, X, None, None, None, None, 1.0, True, torch.empty(0, device=DEV), torch.empty(0, device=DEV), X, X, X, X, None, g, None, None)
    assert not g.any()


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("a", ref.ACTS)
def test_infinities_and_nan_stay_in_their_rows(a, t):
    tx, tw, ty, tz = TYPES[t]
    r = np.random.default_rng(8)
    X, W, Wu = values(r, (70, 100), tx), values(r, (100, 72), tw, 0.1), values(r, (100, 72), tw, 0.1)
    X[3, 99], X[40, 0], X[69, 5] = np.nan, np.inf, -np.inf
    with np.errstate(all="ignore"):
        y = ref.act(X @ W, a)
        h = y * (X @ Wu)
    Y, Hh = out(70, 72, ty), out(70, 72, ty)
    sg.sgnn_linear_fwd(ctx(), dev(X, tx), dev(W, tw), None, ACT[a], flags(t), Y)
    sg.sgnn_glu_fwd(ctx(), dev(X, tx), dev(W, tw), dev(Wu, tw), None, None, ACT[a], flags(t), Hh)
    for got, want in ((Y, y), (Hh, h)):
        got = got.double().cpu().numpy()
        fine = np.ones(70, bool)
        fine[[3, 40, 69]] = False
        assert np.isfinite(got[fine]).all() and np.abs(got[fine] - want[fine]).max() < 0.05 * np.abs(want[fine]).max()
        assert np.isnan(got[3]).all() and np.array_equal(np.isnan(got[[40, 69]]), np.isnan(want[[40, 69]]))
        assert np.array_equal(np.isposinf(got[[40, 69]]), np.isposinf(want[[40, 69]]))


@pytest.mark.parametrize("a", ref.ACTS)
def test_activations_and_slopes_over_the_whole_line(a):
    # W = 1: Z = X; finite arguments of any size have finite activations and slopes
    z = np.concatenate([[0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3], np.linspace(-30, 30, 2001), [88.0, -88.0, 104.0, -104.0, 1e4, -1e4, 1e20, -1e20, 3e38, -3e38]]).astype(np.float32)
    z = z.astype(np.float64)[:, None]
    one = np.ones((1, 1))
    with np.errstate(all="ignore"):
        y, s = ref.act(z, a), ref.act_grad(np.clip(z, -1e9, 1e9), a)
    Y, D, dB = out(len(z), 1, F32), out(len(z), 1, F32), None
    sg.sgnn_linear_fwd(ctx(), dev(z, F32), dev(one, F32), None, ACT[a], 0, Y)
    sg.sgnn_linear_bwd(ctx(), dev(z, F32), dev(one, F32), dev(z, F32), ACT[a], 0, dev(np.ones_like(z), F32), D, None, dB)
    Y, D = Y.double().cpu().numpy(), D.double().cpu().numpy()
    assert np.isfinite(Y).all() and np.isfinite(D).all()
    assert (np.abs(Y - y) <= ref.A * np.maximum(np.abs(z), 1)).all() and (np.abs(D - s) <= ref.A * np.minimum(np.maximum(np.abs(z), 1), 64)).all()
    n = dev(np.full((1, 1), np.nan), F32)
    sg.sgnn_linear_bwd(ctx(), n, dev(one, F32), n, ACT["none" if a == "none" else a], 0, dev(one, F32), n2 := out(1, 1, F32), None, None)
    assert a == "none" or bool(torch.isnan(n2).all())


def _block(t, M=300, d=96, f=200, seed=5):
    tx, tw, _, _ = TYPES[t]
    r = np.random.default_rng(seed)
    v = dict(x=values(r, (M, d), tx), wg=values(r, (d, f), tw, d ** -0.5), wu=values(r, (d, f), tw, d ** -0.5), wd=values(r, (f, d), tw, f ** -0.5), dy=values(r, (M, d), tx, 0.1),
             dn=values(r, (M, d), tx, 0.1))
    v = {k: dev(a, tx if k in ("x", "dy", "dn") else tw) for k, a in v.items()}
    v["g"] = [vec(1 + 0.2 * r.standard_normal(d)) for _ in range(4)]
    return v


def _run_block(c, v, t, stream=None):
    """A whole gated block with its norms, forward and backward: x -> norm -> gated product -> product -> norm, scale, add -> norm."""
    x, (g0, g1, sc, g2), fl, e = v["x"], v["g"], flags(t), 1e-6
    M, d = x.shape
    f = v["wg"].shape[1]
    new = lambda rows, cols: torch.empty((rows, cols), dtype=x.dtype, device=DEV)      # noqa: E731
    row = lambda: torch.empty(M, device=DEV)      # noqa: E731
    col = lambda n: torch.empty(n, device=DEV)      # noqa: E731
    o = v.setdefault("o", dict(n=new(M, d), i0=row(), h=new(M, f), g=new(M, f), u=new(M, f), z=new(M, d), y=new(M, d), n2=new(M, d), i1=row(), i2=row(), dx=new(M, d), dz=new(M, d),
                               dh=new(M, f), dn=new(M, d), dwg=new(d, f), dwu=new(d, f), dwd=new(f, d), dg0=col(d), dg1=col(d), dsc=col(d), dg2=col(d), dxx=new(M, d)))
    kw = dict(stream=stream)
    sg.sgnn_block_norm_fwd(c, x, None, None, None, None, g0, 1.0, False, e, None, o["n"], None, o["i0"], **kw)
    sg.sgnn_glu_fwd(c, o["n"], v["wg"], v["wu"], None, None, ACT["silu"], fl, o["h"], G=o["g"], U=o["u"], **kw)
    sg.sgnn_linear_fwd(c, o["h"], v["wd"], None, ACT["none"], fl, o["z"], **kw)
    sg.sgnn_block_norm_fwd(c, x, o["z"], None, g1, sc, g2, 1.0, True, e, o["y"], o["n2"], o["i1"], o["i2"], **kw)
    sg.sgnn_block_norm_bwd(c, o["z"], o["y"], None, g1, sc, g2, 1.0, True, o["i1"], o["i2"], v["dy"], v["dn"], o["dx"], o["dz"], None, o["dg1"], o["dsc"], o["dg2"], **kw)
    sg.sgnn_linear_bwd(c, o["h"], v["wd"], None, ACT["none"], fl, o["dz"], o["dh"], o["dwd"], None, **kw)
    sg.sgnn_glu_bwd(c, o["n"], v["wg"], v["wu"], o["g"], o["u"], ACT["silu"], fl, o["dh"], o["dn"], o["dwg"], o["dwu"], **kw)
    sg.sgnn_block_norm_bwd(c, None, x, None, None, None, g0, 1.0, False, None, o["i0"], o["dx"], o["dn"], o["dxx"], None, dgamma_pre=o["dg0"], **kw)
    return o


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_a_whole_block_forward_and_backward(t):
    v = _block(t)
    o = _run_block(ctx(), v, t)
    p = {k: v[k].double().cpu().requires_grad_() for k in ("x", "wg", "wu", "wd")}
    g = [a.double().cpu().requires_grad_() for a in v["g"]]
    norm = lambda a, s: a * torch.rsqrt((a * a).mean(1, keepdim=True) + 1e-6) * s      # noqa: E731
    n = norm(p["x"], g[0])
    gg = n @ p["wg"]
    z = (gg * torch.sigmoid(gg) * (n @ p["wu"])) @ p["wd"]
    y = p["x"] + g[2] * norm(z, g[1])
    n2 = norm(y, g[3])
    torch.autograd.backward([y, n2], [v["dy"].double().cpu(), v["dn"].double().cpu()])
    # relative to the 2-norm.  fp32: chains of under twenty kernels of 1e-6 each; bfloat16: some ten roundings of 2^-8 at most on the way, of
    # independent signs (rms 2^-9 each): sqrt(10) 2^-9 < 0.0065, twice that as the bar
    bar = 2e-5 if t == "fp32" else 0.013
    for k, want in (("y", y), ("n2", n2), ("dxx", p["x"].grad), ("dwg", p["wg"].grad), ("dwu", p["wu"].grad), ("dwd", p["wd"].grad), ("dg0", g[0].grad), ("dg1", g[1].grad),
                    ("dsc", g[2].grad), ("dg2", g[3].grad)):
        want = want.detach()
        assert float((o[k].double().cpu() - want).norm() / want.norm()) < bar, k


@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_a_captured_block_replays(t):
    # two graphs of one context, replayed in turn on one stream, with the program's own eager work between them
    c = sg.Context(0)
    c.reserve_ffn(400, 128, 256)
    vs = [_block(t, seed=5), _block(t, M=257, d=104, f=136, seed=6)]
    want = [{k: a.clone() for k, a in _run_block(c, v, t).items()} for v in vs]
    torch.cuda.synchronize()
    graphs = []
    for v in vs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _run_block(c, v, t)
        graphs.append(g)
    for _ in range(3):
        for v, g, w in zip(vs, graphs, want):
            for a in v["o"].values():
                a.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(v["o"][k], w[k]) for k in w)
            _run_block(c, _block(t, M=50, d=32, f=40), t)
    c.close()


def test_a_stream_of_its_own():
    v, s = _block("bf16"), torch.cuda.Stream()
    want = {k: a.clone() for k, a in _run_block(ctx(), v, "bf16").items()}
    c = sg.Context(0)
    c.reserve_ffn(400, 128, 256)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        o = _run_block(c, v, "bf16", stream=s)
    s.synchronize()
    assert all(torch.equal(o[k], want[k]) for k in want)
    c.close()


def test_refusals():
    c = ctx()
    X, W, Y, b = (torch.zeros(s, device=DEV) for s in ((8, 16), (16, 24), (8, 24), (24,)))
    h = lambda a: a.to(BF16)      # noqa: E731

    def refused(code, f, *a, **k):
        with pytest.raises(sg.SgnnError) as e:
            f(*a, **k)
        assert e.value.code == code, e.value
    refused(-1, sg.sgnn_linear_fwd, c, X, W, b, 5, 0, Y)                                        # no such activation
    refused(-1, sg.sgnn_linear_fwd, c, X, W, b, -1, 0, Y)
    refused(-1, sg.sgnn_linear_fwd, c, X, W, b, 0, sg.SGNN_RELU, Y)                             # another call's flag
    refused(-1, sg.sgnn_linear_fwd, c, X, W[:15], b, 0, 0, Y)                                   # shapes
    refused(-1, sg.sgnn_linear_fwd, c, X, W, b, 0, 0, Y[:7])
    refused(-1, sg.sgnn_linear_fwd, c, X, W, b, 0, 0, Y, R=Y[:, :23])
    refused(-1, sg.sgnn_linear_fwd, c, X, W, b, 0, 0, Y, Z=Y)                                   # one matrix for two results
    refused(-1, sg.sgnn_linear_fwd, c, X, torch.zeros((16, 0), device=DEV), None, 0, 0, torch.zeros((8, 0), device=DEV))
    refused(-3, sg.sgnn_linear_fwd, c, h(X), W, b, 0, 0, Y)                                     # bfloat16 without its flag
    refused(-3, sg.sgnn_linear_bwd, c, X, W, Y, 1, 0, Y, None, h(W), None)
    refused(-1, sg.sgnn_linear_bwd, c, X, W, None, 1, 0, Y, None, torch.zeros_like(W), None)   # no Z to take the slope at
    refused(-1, sg.sgnn_linear_bwd, c, X, W, Y, 1, 0, Y, X, None, None)                         # dX over X
    refused(-1, sg.sgnn_glu_fwd, c, X, W, W[:, :23], None, None, 4, 0, Y)
    refused(-1, sg.sgnn_glu_fwd, c, X, W, W, None, None, 4, 0, Y, G=Y)
    D = torch.zeros_like(W)
    refused(-1, sg.sgnn_glu_bwd, c, X, W, W, Y, Y, 4, 0, Y, None, D, D)
    with pytest.raises(ValueError):
        sg.sgnn_linear_fwd(c, X, W, b[:23], 0, 0, Y)
    with pytest.raises(TypeError):
        sg.sgnn_linear_fwd(c, X.double(), W, b, 0, 0, Y)
    with pytest.raises(TypeError):
        sg.sgnn_linear_fwd(c, X.t(), W, b, 0, 0, Y)
    n = torch.zeros(8, device=DEV)
    bn = lambda *a, **k: refused(-1, sg.sgnn_block_norm_fwd, c, *a, **k)      # noqa: E731
    bn(X, X.clone(), torch.zeros((8, 2), device=DEV), None, None, None, 1.0, True, 1e-6, torch.zeros_like(X), None)              # gate of two columns
    bn(X, X.clone(), None, torch.ones(16, device=DEV), None, None, 1.0, False, 1e-6, torch.zeros_like(X), None)                  # scale of no norm
    bn(X, X.clone(), None, None, None, None, 1.0, True, -1.0, torch.zeros_like(X), None)
    bn(X, X.clone(), None, None, None, None, 1.0, True, float("nan"), torch.zeros_like(X), None)
    bn(X, None, None, None, torch.ones(16, device=DEV), None, 1.0, False, 1e-6, None, torch.zeros_like(X))
    bn(X, X.clone(), None, None, None, None, 1.0, False, 1e-6, torch.zeros_like(X), None, n)
    bn(X, X.clone(), None, None, None, None, 1.0, True, 1e-6, None, None)
    wide = torch.zeros((2, 16385), device=DEV)
    refused(-3, sg.sgnn_block_norm_fwd, c, wide, wide.clone(), None, None, None, None, 1.0, True, 1e-6, torch.zeros_like(wide), None)
    refused(-1, sg.sgnn_block_norm_bwd, c, X, None, None, None, None, None, 1.0, True, n, None, None, X, X.clone(), None)        # no Y for the second norm
    refused(-1, sg.sgnn_block_norm_bwd, c, X, None, None, None, None, None, 1.0, True, None, None, X.clone(), None, X.clone(), None)
    small = sg.Context(0)
    refused(-2, sg.sgnn_linear_bwd, small, X, W, Y, 1, 0, Y, X.clone(), D, None)                # nothing reserved
    small.close()


def test_outputs_over_inputs_are_refused():
    c = ctx()
    q = lambda: torch.zeros((16, 16), device=DEV)      # noqa: E731
    X, W, V, Z, G, dY, Y, D = (q() for _ in range(8))

    def refused(f, *a, **k):
        with pytest.raises(sg.SgnnError) as e:
            f(*a, **k)
        assert e.value.code == -1, e.value
    for y, z in ((W, None), (X, None), (Y, W), (Y, X), (Y, Y)):
        refused(sg.sgnn_linear_fwd, c, X, W, None, 1, 0, y, Z=z)
    refused(sg.sgnn_linear_fwd, c, X, W, None, 1, 0, Y, R=Z, Z=Z)
    for h, g, u in ((V, None, None), (Y, V, None), (Y, None, W), (Y, Z, Z)):
        refused(sg.sgnn_glu_fwd, c, X, W, V, None, None, 4, 0, h, G=g, U=u)
    for dx, dw in ((W, None), (Z, None), (dY, None), (D, D), (None, W), (None, X), (None, dY), (None, Z)):
        refused(sg.sgnn_linear_bwd, c, X, W, Z, 1, 0, dY, dx, dw, None)
    for dx, dw, dv in ((V, None, None), (G, None, None), (None, V, None), (None, None, W), (None, D, D), (D, None, D)):
        refused(sg.sgnn_glu_bwd, c, X, W, V, Z, G, 4, 0, dY, dx, dw, dv)
    sg.sgnn_linear_fwd(c, X, X, None, 1, 0, Y, R=X)          # one matrix for several inputs is fine
    sg.sgnn_linear_bwd(c, X, X, X, 1, 0, X, D, Y, None)
