"""The operators of a feed-forward block, as cases to be timed and compared with their plain forms.

Operators:
  linear  Y = act(X W + b) + R, and its backward pass from the kept Z = X W + b
  glu     H = act(X Wg + bg) * (X Wu + bu), and its backward pass from the kept G = X Wg + bg and U = X Wu + bu
  norm    y = alpha x + s * sigmoid(gate) * gamma_post * n(z), N = gamma_pre * n(y), n(v) = v / sqrt(mean v^2 + eps), and its
          backward pass from the kept y and the two rows of 1 / sqrt(mean + eps)
Directions: "infer" (forward, nothing kept), "fwd" (forward of a training step, what the backward pass needs is kept), "bwd".
Types: everything fp32, or activations, weights and their gradients bfloat16; vectors (biases, scales and their gradients) are fp32.
Rows are the vertices of a mini-batch (1 k to 2^20 in this repository's configurations) or, when a trained block answers for single
vertices, one to a few tens; widths 16 to 5632.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
NORM_GRADIENTS = ("dx", "dz", "dgate", "dgamma_post", "dscale", "dgamma_pre")


def listed():
    return [
        # one vertex through the widening product of a block: latency and the bytes of W
        dict(name="linear_token_bf16", op="linear", dir="infer", rows=1, d=1024, f=4096, act="gelu", bias=True, res=False, bf16=True),
        # a few vertices through the narrowing product, residual added
        dict(name="linear_few_bf16", op="linear", dir="infer", rows=24, d=4096, f=1024, act="none", bias=True, res=True, bf16=True),
        # a training step's forward product on a mini-batch of the medium graph in fp32
        dict(name="linear_fwd_medium_fp32", op="linear", dir="fwd", rows=32768, d=256, f=256, act="relu", bias=True, res=True, bf16=False),
        # its backward pass on a mini-batch of the large graph, bfloat16
        dict(name="linear_bwd_large_bf16", op="linear", dir="bwd", rows=262144, d=256, f=256, act="gelu", bias=True, res=False, bf16=True),
        # a few vertices through both projections of a gated block
        dict(name="glu_token_bf16", op="glu", dir="infer", rows=4, d=1024, f=2816, act="silu", bias=False, bf16=True),
        # a training step's gated block on a mini-batch of the medium graph in fp32
        dict(name="glu_fwd_medium_fp32", op="glu", dir="fwd", rows=32768, d=256, f=704, act="silu", bias=True, bf16=False),
        # a wide gated block, evaluation: the matrix pipe
        dict(name="glu_infer_wide_bf16", op="glu", dir="infer", rows=8192, d=2048, f=5632, act="silu", bias=False, bf16=True),
        # the backward pass of a gated block on half a mini-batch of the large graph, bfloat16
        dict(name="glu_bwd_large_bf16", op="glu", dir="bwd", rows=131072, d=256, f=704, act="silu", bias=False, bf16=True),
        # ragged sizes in fp32
        dict(name="glu_bwd_ragged_fp32", op="glu", dir="bwd", rows=30011, d=200, f=531, act="gelu_tanh", bias=True, bf16=False),
        # a few wide rows: latency
        dict(name="norm_few_bf16", op="norm", dir="infer", rows=8, d=4096, gate="none", post=True, pre=True, bf16=True),
        # backward on a mini-batch of the medium graph in fp32
        dict(name="norm_bwd_medium_fp32", op="norm", dir="bwd", rows=32768, d=256, gate="row", post=True, pre=True, bf16=False),
        # forward of a training step on the largest mini-batch, a gate of its own for every element
        dict(name="norm_fwd_xlarge_bf16", op="norm", dir="fwd", rows=1048576, d=256, gate="full", post=True, pre=True, bf16=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "glu", "glu", "norm"])
    bf16 = rng.random() < 0.5
    way = rng.choice(["infer", "fwd", "bwd"])
    if op == "norm":
        d = rng.choice([64, 128, 256, 512, 1024, 2048, rng.randint(17, 1500), rng.randint(17, 5632)])
        rows = _log(rng, 1, max(2, min(1 << 20, 180000000 // d)))
        return dict(op=op, dir=way, rows=rows, d=d, gate=rng.choice(["none", "row", "full"]), post=rng.random() < 0.7, pre=rng.random() < 0.8, bf16=bf16)
    d, f = (rng.choice([_log(rng, 16, 4096), 8 * _log(rng, 4, 512), 64 * rng.randint(1, 32)]) for _ in range(2))
    # the work of a call stays under that of the widest listed one
    most = min((2.5e11 if bf16 else 3e10) / (2.0 * d * f * (2 if op == "glu" else 1) * (2 if way == "bwd" else 1)), 2e9 / (4.0 * (d + 4 * f)), 1 << 20)
    rows = _log(rng, 1, max(2, int(most)))
    case = dict(op=op, dir=way, rows=rows, d=d, f=f, act=rng.choice(ACTS if op == "linear" else ACTS[1:]), bias=rng.random() < 0.5, bf16=bf16)
    if op == "linear":
        case["res"] = way != "bwd" and rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed((seed * 1000003 + 29) & 0x7FFFFFFFFFFF)
    t = torch.bfloat16 if case["bf16"] else torch.float32
    M, d = case["rows"], case["d"]

    def normal(*shape, scale=1.0, to=t):
        return torch.randn(shape, device=DEV, generator=gen, dtype=torch.float32).mul_(scale).to(to)

    def vector(n, mean, scale):
        return torch.randn(n, device=DEV, generator=gen, dtype=torch.float32) * scale + mean

    def empty(*shape, to=t):
        return torch.empty(shape, dtype=to, device=DEV)

    s = dict(case=case)
    back = case["dir"] == "bwd"
    if case["op"] == "norm":
        s["x"] = normal(M, d)
        # a residual stream of a few units and a block's output of about one
        s["z"] = normal(M, d, scale=1.5)
        s["gate"] = normal(M, {"row": 1, "full": d}[case["gate"]], scale=1.0) if case["gate"] != "none" else None
        s["gamma_post"], s["gamma_pre"], s["scale"] = vector(d, 1.0, 0.1), vector(d, 1.0, 0.1), vector(d, 0.5, 0.1)
        s["alpha"] = 1.0
        if back:
            y, _, a, b = _norm_forward(s, torch.float32)
            s["y"], s["ir_post"], s["ir_pre"] = y.to(t), a, b
            s["dy"], s["dn"] = normal(M, d, scale=1e-3), normal(M, d, scale=1e-3)
            s["out"] = dict(dx=empty(M, d), dz=empty(M, d), dgate=None if s["gate"] is None else empty(*s["gate"].shape),
                            dgamma_post=empty(d, to=torch.float32), dscale=empty(d, to=torch.float32), dgamma_pre=empty(d, to=torch.float32))
        else:
            s["out"] = dict(y=empty(M, d), n=empty(M, d), ir_post=empty(M, to=torch.float32), ir_pre=empty(M, to=torch.float32))
        return s
    f = case["f"]
    s["x"] = normal(M, d)                               # what a norm in front of the block gives
    for k in ("w",) if case["op"] == "linear" else ("wg", "wu"):
        s[k] = normal(d, f, scale=1.0 / math.sqrt(d))
        s["b" + k[1:]] = vector(f, 0.0, 0.1) if case["bias"] else None
    if case["op"] == "linear":
        s["r"] = normal(M, f) if case["res"] else None
    if back:
        s["dy"] = normal(M, f, scale=1e-3)
        for k in ("w",) if case["op"] == "linear" else ("wg", "wu"):
            z = s["x"].float() @ s[k].float()
            if case["bias"]:
                z += s["b" + k[1:]]
            s["z" + k[1:]] = z.to(t)
            del z
            s["d" + k], s["db" + k[1:]] = empty(d, f), empty(f, to=torch.float32) if case["bias"] else None
        s["dx"] = empty(M, d)
    else:
        s["y"] = empty(M, f)
        for k in ("",) if case["op"] == "linear" else ("g", "u"):
            s["z" + k] = empty(M, f) if case["dir"] == "fwd" else None
    return s


# ---------------------------------------------------------------------------------------------- the plain forms

def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return z * (z > 0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1.0 + torch.exp(-z))


def _act_grad(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        th = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + th) + 0.5 * z * (1.0 - th * th) * c * (1.0 + 3.0 * 0.044715 * z * z)
    g = 1.0 / (1.0 + torch.exp(-z))
    return g * (1.0 + z * (1.0 - g))


def _norm_forward(s, p):
    """y, N and both 1 / sqrt(mean + eps), everything in the precision p."""
    case, x, z = s["case"], s["x"].to(p), s["z"].to(p)
    a = torch.rsqrt((z * z).mean(dim=1) + EPS) if case["post"] else torch.ones(z.shape[0], device=z.device, dtype=p)
    b = z * a[:, None] * s["gamma_post"].to(p) if case["post"] else z
    w = 1.0 / (1.0 + torch.exp(-s["gate"].to(p))) if s["gate"] is not None else 1.0
    y = s["alpha"] * x + s["scale"].to(p) * w * b
    c = torch.rsqrt((y * y).mean(dim=1) + EPS)
    return y, y * c[:, None] * s["gamma_pre"].to(p), a, c


def _norm_backward(s, p):
    case, z, y = s["case"], s["z"].to(p), s["y"].to(p)
    dy = s["dy"].to(p)
    out = {}
    if case["pre"]:
        yh = y * s["ir_pre"].to(p)[:, None]
        dn = s["dn"].to(p)
        out["dgamma_pre"] = (dn * yh).sum(dim=0)
        g = dn * s["gamma_pre"].to(p)
        dy = dy + s["ir_pre"].to(p)[:, None] * (g - yh * (g * yh).mean(dim=1, keepdim=True))
    zh = z * s["ir_post"].to(p)[:, None] if case["post"] else z
    b = zh * s["gamma_post"].to(p) if case["post"] else z
    sc = s["scale"].to(p)
    w = 1.0 / (1.0 + torch.exp(-s["gate"].to(p))) if s["gate"] is not None else 1.0
    out["dx"] = s["alpha"] * dy
    out["dscale"] = (dy * w * b).sum(dim=0)
    if s["gate"] is not None:
        dg = dy * sc * b * w * (1.0 - w)
        out["dgate"] = dg.sum(dim=1, keepdim=True) if case["gate"] == "row" else dg
    db = dy * sc * w
    if case["post"]:
        out["dgamma_post"] = (db * zh).sum(dim=0)
        g = db * s["gamma_post"].to(p)
        out["dz"] = s["ir_post"].to(p)[:, None] * (g - zh * (g * zh).mean(dim=1, keepdim=True))
    else:
        out["dz"] = db
    return out


def _plain(s):
    case, p = s["case"], torch.float32
    t = torch.bfloat16 if case["bf16"] else p
    if case["op"] == "norm":
        if case["dir"] == "bwd":
            o = _norm_backward(s, p)
            return {k: o[k].to(t) if k in ("dx", "dz", "dgate") else o[k] for k in NORM_GRADIENTS if k in o}
        y, n, a, c = _norm_forward(s, p)
        o = dict(y=y.to(t))
        if case["pre"]:
            o["n"] = n.to(t)
        if case["dir"] == "fwd":
            o.update({k: v for k, v, used in (("ir_post", a, case["post"]), ("ir_pre", c, case["pre"])) if used})
        return o
    x = s["x"].to(p)
    if case["dir"] != "bwd":
        kept = {}
        for k in ("",) if case["op"] == "linear" else ("g", "u"):
            z = x @ s["w" + k].to(p)
            kept["z" + k] = z + s["b" + k] if case["bias"] else z
        if case["op"] == "linear":
            y = _act(kept["z"], case["act"])
            y = y + s["r"].to(p) if case["res"] else y
        else:
            y = _act(kept["zg"], case["act"]) * kept["zu"]
        return dict(y=y.to(t), **({k: v.to(t) for k, v in kept.items()} if case["dir"] == "fwd" else {}))
    dy = s["dy"].to(p)
    if case["op"] == "linear":
        dz = {"": dy * _act_grad(s["z"].to(p), case["act"])}
    else:
        g, u = s["zg"].to(p), s["zu"].to(p)
        dz = {"g": dy * u * _act_grad(g, case["act"]), "u": dy * _act(g, case["act"])}
    o, dx = {}, 0.0
    for k, v in dz.items():
        o["dw" + k] = (x.t() @ v).to(t)
        if case["bias"]:
            o["db" + k] = v.sum(dim=0)
        dx = dx + v @ s["w" + k].to(p).t()
    o["dx"] = dx.to(t)
    return o


# ---------------------------------------------------------------------------------------------- the framework's calls

_held = {}


def _context(s):
    """The program's one context, with scratch for what this state calls."""
    import paper_2604_02651_amd as sg
    if not _held:
        _held["ctx"] = sg.Context(0)
    case = s["case"]
    _held["ctx"].reserve_ffn(case["rows"], case["d"], case.get("f", case["d"]))
    s["sg"], s["ctx"] = sg, _held["ctx"]
    s["act"] = getattr(sg, "SGNN_ACT_" + case.get("act", "none").upper())
    s["flags"] = sg.SGNN_BF16_MFMA if case["bf16"] else 0


def _framework(s):
    if "ctx" not in s:
        _context(s)
    sg, c, case = s["sg"], s["ctx"], s["case"]
    if case["op"] == "norm":
        o = s["out"]
        post, pre = case["post"], case["pre"]
        gp, gn = s["gamma_post"] if post else None, s["gamma_pre"] if pre else None
        if case["dir"] == "bwd":
            sg.sgnn_block_norm_bwd(c, s["z"], s["y"] if pre else None, s["gate"], gp, s["scale"], gn, s["alpha"], post, s["ir_post"] if post else None,
                                   s["ir_pre"] if pre else None, s["dy"], s["dn"] if pre else None, o["dx"], o["dz"], o["dgate"],
                                   o["dgamma_post"] if post else None, o["dscale"], o["dgamma_pre"] if pre else None)
            return {k: o[k] for k in NORM_GRADIENTS if o[k] is not None and (post or k != "dgamma_post") and (pre or k != "dgamma_pre")}
        keep = case["dir"] == "fwd"
        sg.sgnn_block_norm_fwd(c, s["x"], s["z"], s["gate"], gp, s["scale"], gn, s["alpha"], post, EPS, o["y"], o["n"] if pre else None,
                               o["ir_post"] if keep and post else None, o["ir_pre"] if keep and pre else None)
        return {k: o[k] for k, used in (("y", True), ("n", pre), ("ir_post", keep and post), ("ir_pre", keep and pre)) if used}
    act, fl = s["act"], s["flags"]
    if case["dir"] != "bwd":
        if case["op"] == "linear":
            sg.sgnn_linear_fwd(c, s["x"], s["w"], s["b"], act, fl, s["y"], R=s["r"], Z=s["z"])
            kept = ("z",)
        else:
            sg.sgnn_glu_fwd(c, s["x"], s["wg"], s["wu"], s["bg"], s["bu"], act, fl, s["y"], G=s["zg"], U=s["zu"])
            kept = ("zg", "zu")
        return dict(y=s["y"], **({k: s[k] for k in kept} if case["dir"] == "fwd" else {}))
    if case["op"] == "linear":
        sg.sgnn_linear_bwd(c, s["x"], s["w"], s["z"], act, fl, s["dy"], s["dx"], s["dw"], s["db"])
        names = ("dw", "db", "dx")
    else:
        sg.sgnn_glu_bwd(c, s["x"], s["wg"], s["wu"], s["zg"], s["zu"], act, fl, s["dy"], s["dx"], s["dwg"], s["dwu"], dbg=s["dbg"], dbu=s["dbu"])
        names = ("dwg", "dbg", "dwu", "dbu", "dx")
    return {k: s[k] for k in names if s[k] is not None}


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e, M, d = 2 if case["bf16"] else 4, case["rows"], case["d"]
    if case["op"] == "norm":
        gate = {"none": 0, "row": 1, "full": d}[case["gate"]] * M * e
        pre, post = case["pre"], case["post"]
        if case["dir"] == "bwd":      # z, y, dY, dN and the gate; dX, dZ and the gate's gradient
            return {"bytes": M * d * e * (4 + 2 * pre) + 2 * gate + 4 * M * (pre + post) + 8 * d * (1 + pre + post), "flops": M * d * (6 + 8 * pre + 6 * post)}
        kept = 4 * M * (pre + post) if case["dir"] == "fwd" else 0
        return {"bytes": M * d * e * (3 + pre) + gate + kept + 4 * d * (1 + pre + post), "flops": M * d * (4 + 4 * pre + 4 * post)}
    f, n = case["f"], 1 if case["op"] == "linear" else 2
    vec = 4 * n * f if case["bias"] else 0
    if case["dir"] == "bwd":          # X, W, Z, dY; dX, dW, db
        return {"bytes": e * (2 * M * d + 2 * n * d * f + (n + 1) * M * f) + vec, "flops": 4 * n * M * d * f}
    kept = n * M * f if case["dir"] == "fwd" else 0
    return {"bytes": e * (M * d + n * d * f + M * f * (1 + bool(case.get("res"))) + kept) + vec, "flops": 2 * n * M * d * f}


# ---------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s, D = prepare(case, seed), torch.float64
    up = {k: v.to(D) for k, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    erf_half = lambda v: torch.special.ndtr(v)                                    # noqa: E731  Phi(v) = (1 + erf(v / sqrt 2)) / 2
    inner = lambda v: 2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)    # noqa: E731  (1 + tanh(u)) / 2 = sigmoid(2 u)
    gates = {"none": lambda v: torch.ones_like(v), "relu": lambda v: torch.heaviside(v, torch.zeros_like(v)), "gelu": erf_half,
             "gelu_tanh": lambda v: torch.sigmoid(inner(v)), "silu": torch.sigmoid}

    def slope(v, act):
        g = gates[act](v)
        if act in ("none", "relu"):
            return g
        if act == "gelu":
            return g + v * torch.exp(-0.5 * v ** 2) / math.sqrt(2.0 * math.pi)
        return g + v * g * (1.0 - g) * (1.0 if act == "silu" else 2.0 * math.sqrt(2.0 / math.pi) * (1.0 + 0.134145 * v ** 2))

    if case["op"] == "norm":
        gate = torch.sigmoid(up["gate"]) if s["gate"] is not None else torch.ones((), dtype=D, device=DEV)
        M, d = case["rows"], case["d"]
        gp = up["gamma_post"] if case["post"] else torch.ones(d, dtype=D, device=DEV)
        if case["dir"] != "bwd":
            ra = ((up["z"].square().sum(1) / d + EPS) ** -0.5) if case["post"] else torch.ones(M, dtype=D, device=DEV)
            y = torch.addcmul(s["alpha"] * up["x"], up["scale"] * gate, up["z"] * ra.unsqueeze(1) * gp)
            rc = (y.square().sum(1) / d + EPS) ** -0.5
            o = dict(y=y)
            if case["pre"]:
                o["n"] = up["gamma_pre"] * y * rc.unsqueeze(1)
            if case["dir"] == "fwd":
                if case["post"]:
                    o["ir_post"] = ra
                if case["pre"]:
                    o["ir_pre"] = rc
            return o
        ra = up["ir_post"].unsqueeze(1) if case["post"] else 1.0
        total, o = up["dy"], {}
        if case["pre"]:
            rc = up["ir_pre"].unsqueeze(1)
            h = up["y"] * rc
            o["dgamma_pre"] = torch.einsum("ij,ij->j", up["dn"], h)
            v = up["dn"] * up["gamma_pre"]
            total = total + rc * (v - h * ((v * h).sum(1, keepdim=True) / d))
        h = up["z"] * ra
        o["dx"] = s["alpha"] * total
        o["dscale"] = (total * gate * h * gp).sum(0)
        through = total * up["scale"]
        if s["gate"] is not None:
            v = through * h * gp * gate * (1.0 - gate)
            o["dgate"] = v.sum(1, keepdim=True) if case["gate"] == "row" else v
        v = through * gate
        if case["post"]:
            o["dgamma_post"] = (v * h).sum(0)
            v = v * gp
            o["dz"] = ra * (v - h * ((v * h).sum(1, keepdim=True) / d))
        else:
            o["dz"] = v
        return o
    parts = ("",) if case["op"] == "linear" else ("g", "u")
    if case["dir"] != "bwd":
        z = {}
        for k in parts:
            z[k] = torch.mm(up["x"], up["w" + k])
            if case["bias"]:
                z[k] += up["b" + k]
        first = z[parts[0]]
        y = first * gates[case["act"]](first)
        if case["op"] == "glu":
            y = y * z["u"]
        elif case["res"]:
            y = y + up["r"]
        return dict(y=y, **({"z" + k: v for k, v in z.items()} if case["dir"] == "fwd" else {}))
    first = up["z" + parts[0]]
    dz = {parts[0]: up["dy"] * slope(first, case["act"])}
    if case["op"] == "glu":
        dz["g"] = dz["g"] * up["zu"]
        dz["u"] = up["dy"] * first * gates[case["act"]](first)
    o = {}
    for k in parts:
        o["dw" + k] = torch.mm(up["x"].mT, dz[k])
        if case["bias"]:
            o["db" + k] = dz[k].sum(0)
    o["dx"] = sum(torch.mm(dz[k], up["w" + k].mT) for k in parts)
    return o
