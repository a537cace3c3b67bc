"""Cases that measure the dense operators around a sketch: layer norm of a sum, and a linear layer with its bias,
activation and residual, each with its gradient.

    norm    y = (h - mean h) / sqrt(var h + eps) * w + b over the last axis, h = x + r
    linear  z = x W^T + b,  y = act(z) + r;  act: none, relu, gelu (with erf), silu, or swiglu, where z holds two
            halves and y = silu(first half) * second half + r

A training forward returns what its gradient needs beside y (the norm's mean and 1/sqrt(var + eps), the linear
layer's z).  The gradients: x, r, w and b of the norm; x, W and b of the linear layer.  Every case is a dict of plain
values, the tensors' contents follow from the seed.
"""
import math

import torch

own = False

EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases

def _norm(name, kind, rows, n, x, r, y):
    """x, r (or None) and y: types; parameters have y's."""
    return {"name": name, "kind": kind, "rows": rows, "n": n, "x": x, "r": r, "y": y}


def _linear(name, kind, dt, rows, k, n, act, bias=True, res=False, pre=False):
    return {"name": name, "kind": kind, "dt": dt, "rows": rows, "k": k, "n": n, "act": act, "bias": bias, "res": res,
            "pre": pre}


def listed():
    return [
        # a single target's features before a ranking tower: the smallest serving call, latency
        _norm("norm one row", "norm", 1, 1024, "bf16", None, "bf16"),
        # what a batch's fp32 sketches [128 users, 8 heads, 512] aggregate, added to the bf16 state and normalised
        _norm("norm sketches", "norm", 128 * 8 * 512, 128, "f32", "bf16", "bf16"),
        # rows of an odd width, nothing aligned: features cut out of a concatenation
        _norm("norm odd rows", "norm", 10007, 1001, "bf16", "bf16", "bf16"),
        # the sketches' gradient, with the reduction of the weight's over a quarter of a million rows
        _norm("norm grad sketches", "norm grad", 262147, 128, "f32", "bf16", "bf16"),
        # gradient at a ranking tower's width
        _norm("norm grad wide", "norm grad", 8192, 4096, "bf16", None, "bf16"),
        # one target through a tower's first layer: a matrix read for a single row
        _linear("linear one target", "linear", "bf16", 1, 1024, 4096, "gelu"),
        # a small request's 16 candidates through a wide gated layer: bound by reading the weights
        _linear("linear few targets", "linear", "bf16", 16, 4096, 8192, "swiglu", bias=False),
        # feed-forward layer over the sketches of 128 users in training: thin products, bound by memory
        _linear("linear feed sketches", "linear", "bf16", 128 * 512, 128, 512, "swiglu", pre=True),
        # a tower's projection added to its input over a training batch of targets: bound by the products
        _linear("linear tower", "linear", "bf16", 8192, 4096, 4096, "none", res=True),
        # fp32 training at sizes that nothing divides
        _linear("linear odd fp32", "linear", "f32", 1003, 509, 777, "gelu", res=True, pre=True),
        # a small model's fp32 step: gradients of one user's sketch through its feed-forward layer
        _linear("linear grad fp32", "linear grad", "f32", 512, 128, 512, "gelu"),
        # gradients of a gated layer over a training batch
        _linear("linear grad gated", "linear grad", "bf16", 16384, 1024, 4096, "swiglu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Spread over the logarithm; half of the sizes are multiples of 16, as widths mostly are."""
    n = _log(rng, lo, hi)
    return max(16, n // 16 * 16) if rng.random() < 0.5 else n


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm grad", "linear", "linear", "linear grad"])
        if kind.startswith("norm"):
            y = rng.choice(["bf16", "bf16", "f32"])
            c = _norm("", kind, _log(rng, 1, 600000), _size(rng, 32, 16384), rng.choice(["bf16", "f32"]),
                      rng.choice([None, "bf16", "f32"]), y)
            ok = c["rows"] * c["n"] < 7e7
        else:
            rows = _log(rng, 1, 64) if rng.random() < 0.3 else _log(rng, 64, 200000)
            c = _linear("", kind, rng.choice(["bf16", "bf16", "f32"]), rows, _size(rng, 32, 8192), _size(rng, 32, 8192),
                        rng.choice(["none", "relu", "gelu", "silu", "swiglu"]), bias=rng.random() < 0.7,
                        res=kind == "linear" and rng.random() < 0.4, pre=kind == "linear" and rng.random() < 0.4)
            w = work(c)
            ok = w["flops"] < (2.5e11 if c["dt"] == "bf16" else 4e10) and w["bytes"] < 1e9
        if ok:
            del c["name"]
            return c


def work(case):
    es = {None: 0, "bf16": 2, "f32": 4}
    if case["kind"].startswith("norm"):
        cells, x, r, y = case["rows"] * case["n"], es[case["x"]], es[case["r"]], es[case["y"]]
        if case["kind"] == "norm":  # x, r in, y out, the parameters
            return {"bytes": cells * (x + r + y) + 2 * case["n"] * y, "flops": 8 * cells}
        # x, r, dy and two numbers a row in, dx, dr out, w in, dw and db out
        return {"bytes": cells * (2 * x + 2 * r + y) + 8 * case["rows"] + 3 * case["n"] * y, "flops": 14 * cells}
    e, M, K, N = es[case["dt"]], case["rows"], case["k"], case["n"]
    Z = 2 * N if case["act"] == "swiglu" else N
    if case["kind"] == "linear":  # x, W, b, r in, y and z out
        z = Z if case["pre"] and case["act"] != "none" else 0
        return {"bytes": e * (M * K + Z * K + Z * case["bias"] + M * N * (1 + case["res"]) + M * z), "flops": 2.0 * M * K * Z}
    z = 0 if case["act"] == "none" else M * Z
    # dy, z, x, W in, dx, dW, db out
    return {"bytes": e * (M * N + z + 2 * M * K + 2 * Z * K + Z * case["bias"]), "flops": 4.0 * M * K * Z}


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    s = {"case": case}
    if case["kind"].startswith("norm"):
        rows, n = case["rows"], case["n"]
        # sums over histories of different lengths: rows of different sizes, some features louder, an offset
        loud = torch.exp(0.5 * normal(n))
        size = torch.exp(0.5 * normal(rows, 1))
        x = normal(rows, n).mul_(loud).add_(0.5).mul_(size)
        s["x"] = x.to(DTYPES[case["x"]])
        s["r"] = normal(rows, n).to(DTYPES[case["r"]]) if case["r"] else None
        y = DTYPES[case["y"]]
        s["w"], s["b"] = (1 + 0.1 * normal(n)).to(y), (0.1 * normal(n)).to(y)
        if case["kind"] == "norm grad":
            s["dy"] = normal(rows, n).to(y)
            _, s["stats"] = _norm_plain(s)  # as the forward left it
        return s
    M, K, N, dt, act = case["rows"], case["k"], case["n"], DTYPES[case["dt"]], case["act"]
    Z = 2 * N if act == "swiglu" else N
    s["x"] = normal(M, K).to(dt)
    s["w"] = normal(Z, K).div_(math.sqrt(K)).to(dt)
    s["b"] = (0.2 * normal(Z)).to(dt) if case["bias"] else None
    s["r"] = normal(M, N).to(dt) if case["res"] else None
    if case["kind"] == "linear grad":
        s["dy"] = normal(M, N).to(dt)
        s["z"] = None if act == "none" else _z_plain(s).to(dt)  # as the forward left it
    return s


# ------------------------------------------------------------ plain forms

def _norm_plain(s):
    h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
    mean = h.mean(-1, keepdim=True)
    h = h - mean
    rstd = 1.0 / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS)
    y = h.mul_(rstd) * s["w"].float() + s["b"].float()
    return y.to(s["w"].dtype), torch.cat([mean, rstd], -1)


def _norm_grad_plain(s):
    h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
    mean, rstd = s["stats"][:, :1], s["stats"][:, 1:]
    xh = (h - mean) * rstd
    dy = s["dy"].float()
    dw, db = (dy * xh).sum(0), dy.sum(0)
    g = dy * s["w"].float()
    dh = (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True)) * rstd
    out = {"dx": dh.to(s["x"].dtype), "dw": dw.to(s["w"].dtype), "db": db.to(s["w"].dtype)}
    if s["r"] is not None:
        out["dr"] = dh.to(s["r"].dtype)
    return out


def _z_plain(s):
    z = s["x"].float() @ s["w"].float().T
    return z if s["b"] is None else z.add_(s["b"].float())


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "swiglu":
        a, u = z.chunk(2, -1)
        return a / (1 + torch.exp(-a)) * u
    return z


def _act_grad(dy, z, act):
    if act == "relu":
        return dy * (z > 0)
    if act == "gelu":
        return dy * (0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return dy * (p + z * p * (1 - p))
    if act == "swiglu":
        a, u = z.chunk(2, -1)
        p = 1 / (1 + torch.exp(-a))
        return torch.cat([dy * u * (p + a * p * (1 - p)), dy * a * p], -1)
    return dy


def _linear_plain(s):
    case, dt = s["case"], s["x"].dtype
    z = _z_plain(s)
    y = _act(z, case["act"])
    out = {"y": (y if s["r"] is None else y + s["r"].float()).to(dt)}
    if case["pre"] and case["act"] != "none":
        out["z"] = z.to(dt)
    return out


def _linear_grad_plain(s):
    dt = s["x"].dtype
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = _act_grad(dz, s["z"].float(), s["case"]["act"])
    out = {"dx": (dz @ s["w"].float()).to(dt), "dw": (dz.T @ s["x"].float()).to(dt)}
    if s["b"] is not None:
        out["db"] = dz.sum(0).to(dt)
    return out


def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2609_08443_gb300 import binding as b

        case = s["case"]
        if kind == "norm":
            return {"y": b.sa_layer_norm_fwd(s["x"], s["w"], s["b"], residual=s["r"], eps=EPS, dtype=s["w"].dtype)}
        if kind == "norm grad":
            dx, dr, dw, db = b.sa_layer_norm_bwd(s["dy"], s["x"], s["stats"], s["w"], residual=s["r"])
            out = {"dx": dx, "dw": dw, "db": db}
            return out if s["r"] is None else {**out, "dr": dr}
        if kind == "linear":
            pre = case["pre"] and case["act"] != "none"
            got = b.sa_linear_fwd(s["x"], s["w"], s["b"], activation=case["act"], residual=s["r"], want_pre=pre)
            return {"y": got[0], "z": got[1]} if pre else {"y": got}
        dx, dw, db = b.sa_linear_bwd(s["dy"], s["x"], s["w"], s["z"], activation=case["act"], want_db=s["b"] is not None)
        return {"dx": dx, "dw": dw} if s["b"] is None else {"dx": dx, "dw": dw, "db": db}
    if kind == "norm":
        return {"y": _norm_plain(s)[0]}
    if kind == "norm grad":
        return _norm_grad_plain(s)
    return _linear_plain(s) if kind == "linear" else _linear_grad_plain(s)


# ------------------------------------------------------------ in 64 bits

def _f64(t, grad=False):
    return None if t is None else t.double().requires_grad_(grad)


def _activation64(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":  # z times the normal distribution's share below z
        return z * torch.special.erfc(-z / math.sqrt(2.0)) / 2
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "swiglu":
        n = z.shape[-1] // 2
        return z[..., :n] * torch.sigmoid(z[..., :n]) * z[..., n:]
    return z


def exact(case, seed):
    """Forward from the definition, gradients from it by differentiation."""
    s = prepare(case, seed)
    if case["kind"].startswith("norm"):
        grad = case["kind"] == "norm grad"
        x, r, w, b = (_f64(s[k], grad) for k in ("x", "r", "w", "b"))
        h = x if r is None else x + r
        var, mean = torch.var_mean(h, -1, correction=0, keepdim=True)
        y = w * (h - mean) / (var + EPS).sqrt() + b
        if not grad:
            return {"y": y}
        y.backward(s["dy"].double())
        out = {"dx": x.grad, "dw": w.grad, "db": b.grad}
        return out if r is None else {**out, "dr": r.grad}
    act = case["act"]
    x, w, b, r = (_f64(s[k]) for k in ("x", "w", "b", "r"))
    if case["kind"] == "linear":
        z = torch.einsum("mk,zk->mz", x, w)
        z = z if b is None else z + b
        y = _activation64(z, act)
        out = {"y": y if r is None else y + r}
        return {**out, "z": z} if case["pre"] and act != "none" else out
    dz = s["dy"].double()
    if act != "none":
        z = _f64(s["z"], True)
        _activation64(z, act).backward(dz)
        dz = z.grad
    out = {"dx": torch.einsum("mz,zk->mk", dz, w), "dw": torch.einsum("mz,mk->zk", dz, x)}
    return out if b is None else {**out, "db": dz.sum(0)}
