"""The feed-forward operators in 64 bits, written out from their formulas with numpy, and how far a correct fp32 / bfloat16 evaluation may be off.

Bounds are per element.  H = 2^-8 (bfloat16) is the largest relative error of one rounding, E = 2^-24 that of an fp32 operation.  A sum of K products is off
by at most (K + 4) E times the sum of their magnitudes, in whichever order it is added up (4: what the split of fp32 operands into three bfloat16
parts leaves out, under 2 E, and its parts' own sums; two fp16 parts leave out up to 8 E of a product, in kernels that sum in the pipe's blocks of 16 products, one
rounding each: (K / 16 + 8) E, which is less from K = 5 on).  An activation of one argument is evaluated to within A = 2^-20 of max(|z|, 1): some ten fp32
operations, each E, and a hardware exponential and reciprocal, an ulp each, with arguments up to 20 and more where the result is not 0.
"""
import numpy as np
from scipy.special import erf

H, E, A = 2.0 ** -8, 2.0 ** -24, 2.0 ** -20
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
SLOPE = 1.13      # the largest |act'| of any of them
CURVE = 1.2       # the largest |act''| (ReLU apart, which is taken at the same z on both sides)


def act(z, name):
    if name == "none":
        return z
    if name == "relu":
        return np.where(np.isnan(z), z, np.maximum(z, 0))
    if name == "gelu":
        return 0.5 * z * (1 + erf(z / np.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))
    return z / (1 + np.exp(-z))


def act_grad(z, name):
    if name == "none":
        return np.ones_like(z)
    if name == "relu":
        return np.where(np.isnan(z), z, (z > 0).astype(np.float64))
    if name == "gelu":
        return 0.5 * (1 + erf(z / np.sqrt(2))) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if name == "gelu_tanh":
        c = np.sqrt(2 / np.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + np.exp(-z))
    return s * (1 + z * (1 - s))


def round_bf16(x):
    """To nearest even, as float64."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32)
    return np.where(np.isfinite(x), r.view(np.float32), np.asarray(x, np.float32)).astype(np.float64)


def product(X, W, b=None):
    """X W + b and the bound of an fp32 evaluation."""
    z = X @ W
    e = (X.shape[1] + 4) * E * (np.abs(X) @ np.abs(W))
    if b is not None:
        z = z + b
        e = e + E * (np.abs(z) + np.abs(b))
    return z, e


def linear_fwd(X, W, b, a, R=None):
    """(Y, bound), (Z, bound)"""
    z, ez = product(X, W, b)
    y = act(z, a)
    ey = SLOPE * ez + A * np.maximum(np.abs(z), 1) * (a not in ("none", "relu"))
    if R is not None:
        y = y + R
        ey = ey + E * (np.abs(y) + np.abs(R))
    return (y, ey), (z, ez)


def glu_fwd(X, Wg, Wu, bg, bu, a):
    g, eg = product(X, Wg, bg)
    u, eu = product(X, Wu, bu)
    f = act(g, a)
    ef = SLOPE * eg + A * np.maximum(np.abs(g), 1)
    return (f * u, ef * np.abs(u) + np.abs(f) * eu + ef * eu + E * np.abs(f * u)), (g, eg), (u, eu)


def _back(X, Ws, ds, es, b16):
    """dX, dWs, dbs with bounds from the gradients ds of the pre-activations (error es before any rounding)."""
    M, N = ds[0].shape
    dX = eX = 0
    dWs, dbs = [], []
    for W, d, e in zip(Ws, ds, es):
        db, eb = d.sum(0), e.sum(0) + (M + 4) * E * np.abs(d).sum(0)
        dbs.append((db, eb))
        ed = e + (H * (np.abs(d) + e) if b16 else 0)
        dWs.append((X.T @ d, np.abs(X).T @ ed + (M + 4) * E * (np.abs(X).T @ np.abs(d))))
        dX = dX + d @ W.T
        eX = eX + ed @ np.abs(W).T + (len(Ws) * N + 4) * E * (np.abs(d) @ np.abs(W).T)
    return (dX, eX), dWs, dbs


def linear_bwd(X, W, Z, a, dY, b16):
    s = act_grad(Z, a)
    d = dY * s
    e = np.abs(dY) * (A * np.maximum(np.abs(Z), 1) * (a not in ("none", "relu"))) + 2 * E * np.abs(d)
    return _back(X, [W], [d], [e], b16)


def glu_bwd(X, Wg, Wu, G, U, a, dH, b16):
    s, f = act_grad(G, a), act(G, a)
    ea = A * np.maximum(np.abs(G), 1)
    ds = [dH * U * s, dH * f]
    es = [np.abs(dH * U) * ea + 3 * E * np.abs(ds[0]), np.abs(dH) * ea + 2 * E * np.abs(ds[1])]
    return _back(X, [Wg, Wu], ds, es, b16)


def rmsnorm(v, eps):
    ir = 1 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
    return v * ir, ir[:, 0]


def block_norm_fwd(X, Z, gate=None, gamma_post=None, scale=None, gamma_pre=None, alpha=1.0, post=True, eps=1e-6):
    """Y, N, ir_post, ir_pre"""
    y, ir_post = alpha * X, None
    if Z is not None:
        b = Z
        if post:
            b, ir_post = rmsnorm(Z, eps)
            b = b * (1 if gamma_post is None else gamma_post)
        w = 1 if gate is None else 1 / (1 + np.exp(-gate))
        y = y + (1 if scale is None else scale) * w * b
    n, ir_pre = rmsnorm(y, eps)
    return y, n * (1 if gamma_pre is None else gamma_pre), ir_post, ir_pre


def block_norm_bwd(Z, Y, ir_post, ir_pre, dY, dN, gate=None, gamma_post=None, scale=None, gamma_pre=None, alpha=1.0, post=True):
    """dict of dX, dZ, dgate, dgamma_post, dscale, dgamma_pre from the kept Y, Z and inverse roots"""
    o, t = {}, 0.0 if dY is None else dY
    if dN is not None:
        yh = Y * ir_pre[:, None]
        g = dN * (1 if gamma_pre is None else gamma_pre)
        o["dgamma_pre"] = (dN * yh).sum(0)
        t = t + ir_pre[:, None] * (g - yh * (g * yh).mean(1, keepdims=True))
    o["dX"] = alpha * t
    if Z is None:
        return o
    zh = Z * ir_post[:, None] if post else Z
    b = zh * (1 if gamma_post is None else gamma_post)
    w = np.ones_like(Z[:, :1]) if gate is None else 1 / (1 + np.exp(-gate))
    s = 1 if scale is None else scale
    o["dscale"] = (t * w * b).sum(0)
    if gate is not None:
        dg = t * s * b * w * (1 - w)
        o["dgate"] = dg.sum(1, keepdims=True) if gate.shape[1] == 1 and Z.shape[1] > 1 else dg
    v = t * s * w
    if post:
        o["dgamma_post"] = (v * zh).sum(0)
        h = v * (1 if gamma_post is None else gamma_post)
        o["dZ"] = ir_post[:, None] * (h - zh * (h * zh).mean(1, keepdims=True))
    else:
        o["dZ"] = v
    return o
