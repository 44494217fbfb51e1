"""The 64-bit formulas of the feed-forward operators against differences of their forward forms, and the refusals that need no GPU."""
import numpy as np
import pytest

import ffn_ref as ref


def _difference(f, x, dy, h=1e-5):
    """Central differences of sum(f(x) dy)."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = ((f(a) - f(b)) * dy).sum() / (2 * h)
    return g


def _close(a, b):
    # differences: h^2 times a third derivative of order one, and 1e-16 / h from rounding
    assert np.abs(a - b).max() < 1e-7 * max(1.0, np.abs(b).max()), np.abs(a - b).max()


@pytest.mark.parametrize("a", ref.ACTS)
def test_linear_gradients(a):
    r = np.random.default_rng(3)
    X, W, b, dY = r.standard_normal((4, 5)), r.standard_normal((5, 3)), r.standard_normal(3), r.standard_normal((4, 3))
    (dX, _), dW, db = ref.linear_bwd(X, W, X @ W + b, a, dY, False)
    _close(dX, _difference(lambda v: ref.linear_fwd(v, W, b, a)[0][0], X, dY))
    _close(dW[0][0], _difference(lambda v: ref.linear_fwd(X, v, b, a)[0][0], W, dY))
    _close(db[0][0], _difference(lambda v: ref.linear_fwd(X, W, v, a)[0][0], b, dY))


@pytest.mark.parametrize("a", ref.ACTS[1:])
def test_glu_gradients(a):
    r = np.random.default_rng(4)
    X, Wg, Wu, bg, bu, dH = (r.standard_normal(s) for s in ((4, 5), (5, 3), (5, 3), (3,), (3,), (4, 3)))
    (dX, _), dW, db = ref.glu_bwd(X, Wg, Wu, X @ Wg + bg, X @ Wu + bu, a, dH, False)
    f = lambda *p: ref.glu_fwd(*p, a)[0][0]      # noqa: E731
    _close(dX, _difference(lambda v: f(v, Wg, Wu, bg, bu), X, dH))
    _close(dW[0][0], _difference(lambda v: f(X, v, Wu, bg, bu), Wg, dH))
    _close(dW[1][0], _difference(lambda v: f(X, Wg, v, bg, bu), Wu, dH))
    _close(db[0][0], _difference(lambda v: f(X, Wg, Wu, v, bu), bg, dH))
    _close(db[1][0], _difference(lambda v: f(X, Wg, Wu, bg, v), bu, dH))


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate", [None, 1, 6])
def test_block_norm_gradients(gate, post):
    r = np.random.default_rng(5)
    X, Z, dY, dN = (r.standard_normal((4, 6)) for _ in range(4))
    p = dict(gate=None if gate is None else r.standard_normal((4, gate)), gamma_post=r.standard_normal(6) if post else None, scale=r.standard_normal(6),
             gamma_pre=r.standard_normal(6))
    fixed = dict(alpha=0.7, post=post)
    y, n, ip, iq = ref.block_norm_fwd(X, Z, **p, **fixed, eps=1e-3)
    o = ref.block_norm_bwd(Z, y, ip, iq, dY, dN, **p, **fixed)
    both = lambda X, Z, **q: np.stack(ref.block_norm_fwd(X, Z, **q, **fixed, eps=1e-3)[:2])       # noqa: E731
    d = np.stack([dY, dN])
    _close(o["dX"], _difference(lambda v: both(v, Z, **p), X, d))
    _close(o["dZ"], _difference(lambda v: both(X, v, **p), Z, d))
    for k, name in (("gate", "dgate"), ("gamma_post", "dgamma_post"), ("scale", "dscale"), ("gamma_pre", "dgamma_pre")):
        if p[k] is not None:
            _close(o[name], _difference(lambda v: both(X, Z, **{**p, k: v}), p[k], d))


def test_calls_without_a_context_are_refused():
    from paper_2604_02651_amd import binding
    L = binding.lib()
    none = [None] * 16
    assert L.sgnn_ctx_reserve_ffn(None, 1, 1, 1) == -1
    for name, fill in (("sgnn_linear_fwd", [None] * 4 + [0, 0] + none), ("sgnn_linear_bwd", [None] * 4 + [0, 0] + none), ("sgnn_glu_fwd", [None] * 6 + [0, 0] + none),
                       ("sgnn_glu_bwd", [None] * 6 + [0, 0] + none), ("sgnn_block_norm_fwd", none), ("sgnn_block_norm_bwd", none)):
        f = getattr(L, name)
        assert f(*fill[:len(f.argtypes)]) == -1, name
