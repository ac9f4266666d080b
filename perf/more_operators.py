"""What stands between two aggregations of a network and between the clipped gradient and the weight, as cases that can be timed and compared:
the norms around a block with its gate, its residual and their gradients, the gated projection and its gradients, and updates of weights made
orthogonal by Newton-Schulz products.  Every case exists twice: as elementary torch operations in 32 bits, and as calls of the framework."""
import math

import torch

own = False  # true: the framework's calls; false: elementary torch operations

HALF, SINGLE = torch.float16, torch.float32
TYPES = {"f16": HALF, "f32": SINGLE}
# five steps that bring all but the smallest singular values near one, and the classical ones that bring them to one
QUINTIC = (3.4445, -4.775, 2.0315)
CUBIC = (1.5, -0.5, 0.0)
EPS = 1e-5
_hgnn = None


def _framework():
    global _hgnn
    if _hgnn is None:
        import paper_2411_01109_amd
        _hgnn = paper_2411_01109_amd
    return _hgnn


def listed():
    return [
        # the seed vertices of a sampled batch, before their first layer: nothing but latency
        {"name": "norm_seeds", "kind": "norm", "n": 64, "F": 128, "type": "f16", "post": "none", "pre": "rms", "gate": "none", "bias": False, "alpha": 1.0},
        # between two layers of a product graph: the branch's norm and gate of every feature, the sum, the next layer's norm
        {"name": "norm_layer", "kind": "norm", "n": 2400000, "F": 128, "type": "f16", "post": "layer", "pre": "layer", "gate": "feature", "bias": True, "alpha": 1.0},
        # its gradient, with those of all weights
        {"name": "norm_grad", "kind": "norm_grad", "n": 2400000, "F": 128, "type": "f16", "post": "layer", "pre": "layer", "gate": "feature", "bias": True, "alpha": 1.0},
        # a residual stream in fp32 of an odd width in a padded pitch, every element with a gate of its own
        {"name": "norm_grad_rows", "kind": "norm_grad", "n": 99991, "F": 333, "type": "f32", "post": "rms", "pre": "rms", "gate": "rows", "bias": False, "alpha": 0.7},
        # one vertex (token) of a served model: the weights are all that counts
        {"name": "gated_one", "kind": "gated", "n": 1, "K": 1024, "F": 4096, "act": "silu", "trans": False},
        # a few of them at once, by weights with the inputs along their rows, an odd width
        {"name": "gated_few", "kind": "gated", "n": 13, "K": 2048, "F": 5461, "act": "gelu", "trans": True},
        # all vertices of a graph through a narrow layer
        {"name": "gated_layer", "kind": "gated", "n": 233000, "K": 128, "F": 256, "act": "silu", "trans": False},
        # the gradients of a narrow layer whose inputs have an odd width
        {"name": "gated_grad_layer", "kind": "gated_grad", "n": 99991, "K": 100, "F": 200, "act": "gelu", "trans": False},
        # a wide block's step over a large batch: products and nothing else
        {"name": "gated_grad_wide", "kind": "gated_grad", "n": 8192, "K": 2048, "F": 8192, "act": "silu", "trans": True},
        # the weights of a two-layer network of attention over a graph
        {"name": "orth_layers", "kind": "orth", "matrices": "608x64 64x64 64x64 64x42 42x42", "type": "f32", "out": "f32", "steps": 5, "coef": "quintic"},
        # a projection of a wider network, its update stored in fp16
        {"name": "orth_hidden", "kind": "orth", "matrices": "1024x4096", "type": "f32", "out": "f16", "steps": 5, "coef": "quintic"},
        # a large square weight whose gradient is in fp16
        {"name": "orth_large", "kind": "orth", "matrices": "4096x4096", "type": "f16", "out": "f32", "steps": 5, "coef": "quintic"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over their logarithms, odd ones among them; no more work than the largest listed one."""
    kind = rng.choice(("norm", "norm_grad", "gated", "gated_grad", "orth"))
    c = {"kind": kind}
    if kind in ("norm", "norm_grad"):
        c["F"] = F = rng.choice((5, 7, 16, 42, 64, 100, 128, 128, 200, 256, 333, 512, 608, 1000, 2048, 4096, 8191))
        c["n"] = min(_log(rng, 1, 2400000), 150000000 // F)
        c["type"] = rng.choice(("f16", "f32"))
        c["post"], c["pre"] = rng.choice((("none", "rms"), ("none", "layer"), ("rms", "rms"), ("layer", "layer"), ("rms", "none"), ("layer", "rms")))
        c["gate"] = rng.choice(("none", "feature", "rows"))
        c["bias"] = rng.random() < 0.5
        c["alpha"] = rng.choice((1.0, 0.7))
    elif kind in ("gated", "gated_grad"):
        c["n"] = _log(rng, 1, 250000)
        c["K"] = _log(rng, 8, 4096)
        c["F"] = _log(rng, 8, 8192)
        most = 100000000000
        if c["n"] * c["K"] * c["F"] > most:
            c["n"] = max(1, most // (c["K"] * c["F"]))
        c["n"] = max(1, min(c["n"], 400000000 // (c["K"] + c["F"])))
        c["act"] = rng.choice(("silu", "gelu", "sigmoid", "relu"))
        c["trans"] = rng.random() < 0.5
    else:
        left, t = _log(rng, 1000, 60000000000), []
        for _ in range(_log(rng, 1, 24)):
            a, b = _log(rng, 1, 4096), _log(rng, 1, 4096)
            while a * b * min(a, b) > left:
                a, b = max(1, a // 2), max(1, b * 2 // 3)
            left = max(left - a * b * min(a, b), 1000)
            t.append("%dx%d" % (a, b))
        c["matrices"] = " ".join(t)
        c["type"], c["out"] = rng.choice(("f16", "f32")), rng.choice(("f16", "f32"))
        c["coef"] = rng.choice(("quintic", "quintic", "cubic"))
        c["steps"] = rng.choice((5, 5, 6, 8) if c["coef"] == "quintic" else (5, 10))
    return c


# ---------------------------------------------------------------------------------------------------- inputs
class _State:
    pass


def _pitch(n):
    return (n + 7) // 8 * 8


def _empty(rows, cols, dtype):
    return torch.zeros((rows, _pitch(cols)), dtype=dtype, device="cuda")[:, :cols]


def _normal(gen, rows, cols, dtype, sd=1.0):
    """Normals in rows of a pitch that is a multiple of 8: a view of the columns in use."""
    t = torch.empty((rows, _pitch(cols)), dtype=dtype, device="cuda")
    step = max(1, (1 << 27) // _pitch(cols))
    for r in range(0, rows, step):
        t[r:r + step] = torch.randn((min(step, rows - r), _pitch(cols)), generator=gen, device="cuda") * sd
    return t[:, :cols]


def _vector(gen, n, about, sd):
    return about + sd * torch.randn(n, generator=gen, device="cuda")


def _matrices(c):
    return [tuple(int(v) for v in m.split("x")) for m in c["matrices"].split()]


def prepare(case, seed):
    c, s = case, _State()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s.kind = kind = c["kind"]
    s.case, s.workspace = c, None
    if kind in ("norm", "norm_grad"):
        n, F, stream = c["n"], c["F"], TYPES[c["type"]]
        s.Y = _normal(gen, n, F, HALF, 0.8)
        s.post_w = _vector(gen, F, 1.0, 0.2) if c["post"] != "none" else None
        s.post_b = _vector(gen, F, 0.0, 0.1) if c["post"] != "none" and c["bias"] else None
        s.pre_w = _vector(gen, F, 1.0, 0.2) if c["pre"] != "none" else None
        s.pre_b = _vector(gen, F, 0.0, 0.1) if c["pre"] != "none" and c["bias"] else None
        s.gate = _vector(gen, F, 0.5, 0.2) if c["gate"] == "feature" else _normal(gen, n, F, HALF, 0.5) if c["gate"] == "rows" else None
        s.R = _normal(gen, n, F, stream, 1.5) if kind == "norm" else None
        s.H = _empty(n, F, stream) if kind == "norm" else _normal(gen, n, F, stream, 1.7)
        if kind == "norm":
            s.Z = _empty(n, F, HALF) if c["pre"] != "none" else None
        else:
            s.dH = _normal(gen, n, F, stream, 1.0)
            s.dZ = _normal(gen, n, F, HALF, 1.0) if c["pre"] != "none" else None
            s.dR, s.dY = _empty(n, F, stream), _empty(n, F, HALF)
            vector = lambda wanted: torch.zeros(F, device="cuda") if wanted is not None else None  # noqa: E731
            s.dpost_w, s.dpost_b, s.dpre_w, s.dpre_b = vector(s.post_w), vector(s.post_b), vector(s.pre_w), vector(s.pre_b)
            s.dgate = None if s.gate is None else vector(s.gate) if c["gate"] == "feature" else _empty(n, F, HALF)
    elif kind in ("gated", "gated_grad"):
        n, K, F = c["n"], c["K"], c["F"]
        shape = (F, K) if c["trans"] else (K, F)
        s.X = _normal(gen, n, K, HALF)
        s.Wg, s.Wu = (_normal(gen, *shape, HALF, 1 / math.sqrt(K)) for _ in range(2))
        if kind == "gated":
            s.Y = _empty(n, F, HALF)
        else:
            s.dY = _normal(gen, n, F, HALF, 1 / math.sqrt(F))
            s.dX, s.dWg, s.dWu = _empty(n, K, HALF), _empty(*shape, HALF), _empty(*shape, HALF)
    else:
        # sums of a momentum's directions with falling weights, as gradients of weights are, and noise
        s.grads, s.outs = [], []
        for rows, cols in _matrices(c):
            few = max(1, min(rows, cols) // 4)
            a, b = (torch.randn(shape, generator=gen, device="cuda") for shape in ((rows, few), (few, cols)))
            g = (a * torch.linspace(1.0, 0.1, few, device="cuda")) @ b / math.sqrt(few)
            g = (g + 0.5 * torch.randn((rows, cols), generator=gen, device="cuda")).to(TYPES[c["type"]])
            s.grads.append(g)
            s.outs.append(torch.zeros((rows, cols), dtype=TYPES[c["out"]], device="cuda"))
    return s


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _workspace(s, size):
    if s.workspace is None:  # a program's own, kept from step to step
        s.workspace = torch.empty(max(size(), 16), dtype=torch.uint8, device="cuda")
    return s.workspace


def _block(s, h):
    c, kinds = s.case, {"none": h.HGNN_NORM_NONE, "rms": h.HGNN_NORM_RMS, "layer": h.HGNN_NORM_LAYER}
    return dict(post=kinds[c["post"]], post_w=s.post_w, post_b=s.post_b, gate=s.gate, alpha=c["alpha"], pre=kinds[c["pre"]], pre_w=s.pre_w, pre_b=s.pre_b, eps=EPS)


def _own_norm(s):
    h = _framework()
    h.hgnn_residual_norm(s.R, s.Y, s.H, s.Z, **_block(s, h))
    return {"H": s.H, "Z": s.Z}


def _own_norm_grad(s):
    h = _framework()
    ws = _workspace(s, lambda: h.hgnn_residual_norm_grad_workspace(s.case["n"], s.case["F"]))
    h.hgnn_residual_norm_grad(s.H, s.Y, s.dH, s.dZ, s.dR, s.dY, ws, dgate=s.dgate, dpost_w=s.dpost_w, dpost_b=s.dpost_b, dpre_w=s.dpre_w, dpre_b=s.dpre_b,
                              **_block(s, h))
    return {"dR": s.dR, "dY": s.dY, "dgate": s.dgate, "dpost_w": s.dpost_w, "dpost_b": s.dpost_b, "dpre_w": s.dpre_w, "dpre_b": s.dpre_b}


def _act(s, h):
    return {"silu": h.HGNN_SILU, "gelu": h.HGNN_GELU, "sigmoid": h.HGNN_SIGMOID, "relu": h.HGNN_RELU}[s.case["act"]]


def _own_gated(s):
    h, c = _framework(), s.case
    ws = _workspace(s, lambda: h.hgnn_gated_workspace(c["n"], c["K"], c["F"]))
    h.hgnn_gated(s.X, s.Wg, s.Wu, s.Y, act=_act(s, h), trans_w=c["trans"], workspace=ws)
    return s.Y


def _own_gated_grad(s):
    h, c = _framework(), s.case
    ws = _workspace(s, lambda: h.hgnn_gated_grad_workspace(c["n"], c["K"], c["F"]))
    h.hgnn_gated_grad(s.X, s.Wg, s.Wu, s.dY, s.dX, s.dWg, s.dWu, ws, act=_act(s, h), trans_w=c["trans"])
    return {"dX": s.dX, "dWg": s.dWg, "dWu": s.dWu}


def _own_orth(s):
    h, c = _framework(), s.case
    ws = _workspace(s, lambda: h.hgnn_orthogonalize_workspace(s.grads))
    h.hgnn_orthogonalize(s.grads, s.outs, _coefficients(c), ws)
    return s.outs


# ---------------------------------------------------------------------------------------------------- the plain forms
def _coefficients(c):
    return [QUINTIC if c["coef"] == "quintic" else CUBIC] * c["steps"]


def _normed(x, kind):
    """-> (x normed, 1 / its deviation)"""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    r = (x.square().mean(1, keepdim=True) + EPS).rsqrt()
    return x * r, r


def _affine(x, w, b):
    return x * w if b is None else x * w + b


def _plain_norm(s):
    c = s.case
    b = s.Y.float()
    if c["post"] != "none":
        b = _affine(_normed(b, c["post"])[0], s.post_w, s.post_b)
    if s.gate is not None:
        b = b * s.gate.float()
    H = (c["alpha"] * s.R.float() + b).to(s.R.dtype)
    if c["pre"] == "none":
        return {"H": H, "Z": None}
    return {"H": H, "Z": _affine(_normed(H.float(), c["pre"])[0], s.pre_w, s.pre_b).to(HALF)}


def _norm_back(d, w, xh, r, kind):
    u = d * w
    dx = u - xh * (u * xh).mean(1, keepdim=True)
    if kind == "layer":
        dx = dx - u.mean(1, keepdim=True)
    return dx * r


def _plain_norm_grad(s):
    c = s.case
    got = dict.fromkeys(("dR", "dY", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b"))
    e = s.dH.float()
    if c["pre"] != "none":
        xh, r = _normed(s.H.float(), c["pre"])
        d = s.dZ.float()
        e = e + _norm_back(d, s.pre_w, xh, r, c["pre"])
        got["dpre_w"] = (d * xh).sum(0)
        if c["bias"]:
            got["dpre_b"] = d.sum(0)
    got["dR"] = (c["alpha"] * e).to(s.dR.dtype)
    b = s.Y.float()
    if c["post"] != "none":
        xh, r = _normed(b, c["post"])
        b = _affine(xh, s.post_w, s.post_b)
    d = e
    if s.gate is not None:
        got["dgate"] = (e * b).sum(0) if c["gate"] == "feature" else (e * b).to(HALF)
        d = e * s.gate.float()
    if c["post"] != "none":
        got["dpost_w"] = (d * xh).sum(0)
        if c["bias"]:
            got["dpost_b"] = d.sum(0)
        d = _norm_back(d, s.post_w, xh, r, c["post"])
    got["dY"] = d.to(HALF)
    return got


def _activated(g, act):
    """-> (act(g), its derivative)"""
    if act == "relu":
        return g.clamp(min=0.0), (g > 0).to(g.dtype)
    if act == "gelu":
        phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    p = 1.0 / (1.0 + torch.exp(-g))
    return (p, p * (1.0 - p)) if act == "sigmoid" else (g * p, p * (1.0 + g * (1.0 - p)))


def _weights(s):
    Wg, Wu = s.Wg.float(), s.Wu.float()
    return (Wg.t(), Wu.t()) if s.case["trans"] else (Wg, Wu)


def _plain_gated(s):
    X, (Wg, Wu) = s.X.float(), _weights(s)
    return (_activated(X @ Wg, s.case["act"])[0] * (X @ Wu)).to(HALF)


def _plain_gated_grad(s):
    X, (Wg, Wu) = s.X.float(), _weights(s)
    a, da = _activated(X @ Wg, s.case["act"])
    dY = s.dY.float()
    dG, dU = dY * (X @ Wu) * da, dY * a
    dX = (dG @ Wg.t() + dU @ Wu.t()).to(HALF)
    if s.case["trans"]:
        return {"dX": dX, "dWg": (dG.t() @ X).to(HALF), "dWu": (dU.t() @ X).to(HALF)}
    return {"dX": dX, "dWg": (X.t() @ dG).to(HALF), "dWu": (X.t() @ dU).to(HALF)}


def _plain_orth(s):
    outs = []
    for g, o in zip(s.grads, s.outs):
        x = g.float()
        flip = x.shape[0] > x.shape[1]
        x = x.t() if flip else x
        norm = x.double().square().sum().sqrt()
        x = (x / norm).float()
        for a, b, c in _coefficients(s.case):
            A = x @ x.t()
            x = a * x + (b * A + c * (A @ A)) @ x
        outs.append((x.t() if flip else x).to(o.dtype).contiguous())
    return outs


def run(state):
    if own:
        return {"norm": _own_norm, "norm_grad": _own_norm_grad, "gated": _own_gated, "gated_grad": _own_gated_grad, "orth": _own_orth}[state.kind](state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "gated": _plain_gated, "gated_grad": _plain_gated_grad, "orth": _plain_orth}[state.kind](state)


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    if c["kind"] in ("norm", "norm_grad"):
        size = {"f16": 2, "f32": 4}[c["type"]]
        rows = 2 if c["gate"] == "rows" else 0
        pre = 2 if c["pre"] != "none" else 0
        if c["kind"] == "norm":  # R and H, Y, Z
            return {"bytes": c["n"] * c["F"] * (2 * size + 2 + rows + pre), "flops": 14 * c["n"] * c["F"]}
        # dH and dR, dY, H and dZ where there is a norm in front, Y where it is asked for
        reads = size + pre if pre else 0
        Y = 2 if c["post"] != "none" or c["gate"] != "none" else 0
        return {"bytes": c["n"] * c["F"] * (2 * size + 2 + reads + Y + 2 * rows), "flops": 30 * c["n"] * c["F"]}
    if c["kind"] == "gated":
        n, K, F = c["n"], c["K"], c["F"]
        return {"bytes": 2 * (n * K + 2 * K * F + n * F), "flops": 4 * n * K * F}
    if c["kind"] == "gated_grad":
        n, K, F = c["n"], c["K"], c["F"]
        return {"bytes": 2 * (2 * n * K + n * F + 4 * K * F), "flops": 12 * n * K * F}
    size = {"f16": 2, "f32": 4}
    total = {"bytes": 0, "flops": 0}
    for a, b in _matrices(c):
        m, k = min(a, b), max(a, b)
        total["bytes"] += a * b * (size[c["type"]] + size[c["out"]])
        # both symmetric products by half, and the square only where it counts
        total["flops"] += c["steps"] * (m * m * k + (m * m * m if c["coef"] == "quintic" else 0) + 2 * m * m * k)
    return total


# ---------------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] in ("norm", "norm_grad"):
        return _exact_norm(c, s)
    if c["kind"] in ("gated", "gated_grad"):
        return _exact_gated(c, s)
    outs = []
    for g in s.grads:
        x = g.double()
        x = x / torch.sqrt((x * x).sum())
        # the same polynomial of x from either side: x p(x^T x) = p(x x^T) x
        right = x.shape[1] <= x.shape[0]
        for a, b, q in _coefficients(c):
            gram = x.t() @ x if right else x @ x.t()
            p = b * gram + q * gram.matmul(gram)
            p.diagonal().add_(a)
            x = x @ p if right else p @ x
        outs.append(x)
    return outs


def _moments(x, kind):
    """-> (mean, 1 / deviation) of rows"""
    mean = torch.mean(x, 1, True) if kind == "layer" else torch.zeros_like(x[:, :1])
    return mean, 1 / torch.sqrt(((x - mean) ** 2).mean(1, True) + EPS)


def _exact_norm(c, s):
    """Rows in groups, in 64 bits."""
    names = ("H", "Z") if c["kind"] == "norm" else ("dR", "dY", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b")
    rows = {name: [] for name in names}
    wide = lambda v: None if v is None else v.double()  # noqa: E731
    pw, pb, qw, qb = wide(s.post_w), wide(s.post_b), wide(s.pre_w), wide(s.pre_b)
    step = max(1, (1 << 25) // c["F"])
    for r in range(0, c["n"], step):
        part = slice(r, r + step)
        y = s.Y[part].double()
        gate = 1.0 if s.gate is None else s.gate.double() if c["gate"] == "feature" else s.gate[part].double()
        m1, r1 = _moments(y, c["post"])
        branch = y if pw is None else (y - m1) * r1 * pw + (0.0 if pb is None else pb)
        if c["kind"] == "norm":
            h = c["alpha"] * s.R[part].double() + gate * branch
            rows["H"].append(h)
            if qw is not None:
                h = h.to(s.R.dtype).double()  # what is normed is the stream as it is stored
                m2, r2 = _moments(h, c["pre"])
                rows["Z"].append((h - m2) * r2 * qw + (0.0 if qb is None else qb))
            continue
        e = s.dH[part].double()
        if qw is not None:
            h, dz = s.H[part].double(), s.dZ[part].double()
            m2, r2 = _moments(h, c["pre"])
            e = e + _jacobian(dz * qw, (h - m2) * r2, r2, c["pre"])
            rows["dpre_w"].append((dz * (h - m2) * r2).sum(0))
            rows["dpre_b"].append(dz.sum(0))
        rows["dR"].append(c["alpha"] * e)
        rows["dgate"].append((e * branch).sum(0) if c["gate"] == "feature" else e * branch)
        db = e * gate
        if pw is not None:
            hat = (y - m1) * r1
            rows["dpost_w"].append((db * hat).sum(0))
            rows["dpost_b"].append(db.sum(0))
            db = _jacobian(db * pw, hat, r1, c["post"])
        rows["dY"].append(db)
    got = {}
    for name in names:
        wanted = {"Z": qw, "dgate": s.gate, "dpost_w": pw, "dpost_b": pb, "dpre_w": qw, "dpre_b": qb}.get(name, 0)
        summed = name.startswith(("dpost", "dpre")) or (name == "dgate" and c["gate"] == "feature")
        got[name] = None if wanted is None else torch.stack(rows[name]).sum(0) if summed else torch.cat(rows[name])
    return got


def _jacobian(u, hat, r, kind):
    """u times the derivative of the normed row, which is r (1 - hat hat^T / F), without its mean where the norm takes that off"""
    F = hat.shape[1]
    out = u - (u * hat).sum(1, True) / F * hat
    return r * (out - u.sum(1, True) / F) if kind == "layer" else r * out


def _exact_gated(c, s):
    Wg, Wu = s.Wg.double(), s.Wu.double()
    if c["trans"]:
        Wg, Wu = Wg.mT, Wu.mT
    Y, dX, dW = [], [], [0.0, 0.0]
    step = max(1, (1 << 27) // max(c["K"], c["F"]))
    for r in range(0, c["n"], step):
        x = s.X[r:r + step].double()
        g, u = x.matmul(Wg), x.matmul(Wu)
        if c["act"] == "relu":
            slope = torch.heaviside(g, torch.zeros_like(g[:1, :1]))
            value = g * slope
        elif c["act"] == "gelu":
            normal = torch.special.ndtr(g)
            value, slope = g * normal, normal + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        else:
            p = torch.sigmoid(g)
            value, slope = (p, p - p * p) if c["act"] == "sigmoid" else (g * p, p + g * p * torch.sigmoid(-g))
        if c["kind"] == "gated":
            Y.append(value * u)
            continue
        dy = s.dY[r:r + step].double()
        parts = dy * u * slope, dy * value
        dX.append(parts[0].matmul(Wg.mT) + parts[1].matmul(Wu.mT))
        dW = [total + x.mT.matmul(part) for total, part in zip(dW, parts)]
    if c["kind"] == "gated":
        return torch.cat(Y)
    if c["trans"]:
        dW = [w.mT.contiguous() for w in dW]
    return {"dX": torch.cat(dX), "dWg": dW[0], "dWu": dW[1]}
