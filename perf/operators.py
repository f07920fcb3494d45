"""Operators of residual blocks on node embeddings, as cases that can be timed: the root-mean-square norm of rows with the
residual's addition (and its output in 8 bits), the linear layer with bias, activation and residual (and its gradients), and
the clipping of a gradient by its global norm.

``run`` computes an operator in its plain form, with elementary torch operations in fp32 (fp64 for the long sums of the global norm), or,
where ``own`` is true, with this package's calls.  Inputs are made from the seed alone, on the GPU.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
EPS = 1e-6
E4M3_MAX = 448.0
TINY_SCALE = 2.0 ** -126           # the scale of a row of zeros
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"fp32": 4, "bf16": 2, "e4m3": 1}


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # One node scored online through a 256-wide block: launch and latency, nothing else.
        {"name": "norm_one_node", "op": "norm", "rows": 1, "width": 256, "x": "bf16", "y": "bf16", "residual": True},
        # A partition's hidden features (the second configuration's share, 3e5 nodes of 256) between two layers, kept in fp32.
        {"name": "norm_share", "op": "norm", "rows": 300_001, "width": 256, "x": "fp32", "y": "bf16", "residual": True},
        # The rows that an 8-bit product reads, in a wide model.
        {"name": "norm_8bit_wide", "op": "norm8", "rows": 8192, "width": 8192, "x": "bf16", "residual": True, "normalise": True},
        # Activations (or weights, once) to 8 bits without a norm, rows of a width that is no multiple of anything large.
        {"name": "quantize_activations", "op": "norm8", "rows": 100_003, "width": 1004, "x": "bf16", "residual": False, "normalise": False},
        # The gradient of the norm over the same share, joined with the residual's, and the weight's gradient over all rows.
        {"name": "norm_gradient_share", "op": "norm_grad", "rows": 300_001, "width": 256, "h": "fp32", "dy": "bf16", "residual": True},
        # A linear layer for one node: the weight is read once, and that is all.
        {"name": "linear_one_node", "op": "linear", "rows": 1, "n": 4096, "k": 4096, "dtype": "bf16", "act": "gelu", "residual": True, "c": "bf16",
         "keep": False},
        # A hidden layer over the share: tall and narrow, bound by its rows; the pre-activation is kept for the backward pass.
        {"name": "linear_share", "op": "linear", "rows": 300_001, "n": 256, "k": 256, "dtype": "bf16", "act": "relu", "residual": True, "c": "bf16",
         "keep": True},
        # A wide layer in 8 bits: all matrix instructions.
        {"name": "linear_8bit_wide", "op": "linear", "rows": 8192, "n": 8192, "k": 8192, "dtype": "e4m3", "act": "silu", "residual": False, "c": "bf16",
         "keep": False},
        # The gradient with respect to the layer's input, through the activation below it.
        {"name": "linear_dx_wide", "op": "linear_dx", "rows": 8192, "n": 4096, "k": 4096, "act": "gelu", "d": "bf16"},
        # The gradient of the weight and the bias of a hidden layer: a long sum over the share's nodes.
        {"name": "linear_dw_share", "op": "linear_dw", "rows": 300_001, "n": 256, "k": 256},
        # The gradient of a small model: tensors of a few numbers to a few ten thousand.
        {"name": "clip_small_model", "op": "clip", "tensors": 48, "least": 1, "most": 40_000, "bf16": False, "tight": True},
        # The gradient of a large one: 4e8 bytes in tensors of both types.
        {"name": "clip_large_model", "op": "clip", "tensors": 40, "least": 1_000, "most": 16_000_000, "bf16": True, "tight": True},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Rows from one to 3e5, widths from 8 to 8192, odd ones among them (at most 2^26 elements of a norm, 2^37 products of a layer)."""
    op = rng.choice(["norm", "norm8", "norm_grad", "linear", "linear_dx", "linear_dw", "clip"])
    if op == "clip":
        return {"op": op, "tensors": rng.randint(1, 60), "least": _log(rng, 1, 1000), "most": _log(rng, 1000, 4_000_000),
                "bf16": rng.random() < 0.5, "tight": rng.random() < 0.7}

    def width():
        w = _log(rng, 8, 8192)
        return w if rng.random() < 0.4 else max(8, w // 8 * 8)

    rows = _log(rng, 1, 300_000)
    if op in ("norm", "norm8", "norm_grad"):
        w = width()
        c = {"op": op, "rows": min(rows, (1 << 26) // w), "width": w, "residual": rng.random() < 0.6}
        if op == "norm":
            return {**c, "x": rng.choice(["fp32", "bf16"]), "y": rng.choice(["fp32", "bf16"])}
        if op == "norm8":
            normalise = rng.random() < 0.7
            return {**c, "residual": c["residual"] and normalise, "x": rng.choice(["fp32", "bf16"]), "normalise": normalise}
        return {**c, "h": rng.choice(["fp32", "bf16"]), "dy": rng.choice(["fp32", "bf16"])}
    n, k = width(), width()
    c = {"op": op, "rows": max(1, min(rows, (1 << 37) // (n * k))), "n": n, "k": k}
    if op == "linear":
        return {**c, "dtype": rng.choice(["bf16", "e4m3"]), "act": rng.choice(["none", "relu", "gelu", "silu"]), "residual": rng.random() < 0.5,
                "c": rng.choice(["fp32", "bf16"]), "keep": rng.random() < 0.4}
    if op == "linear_dx":
        return {**c, "act": rng.choice(["none", "relu", "gelu", "silu"]), "d": rng.choice(["fp32", "bf16"])}
    return c


def _counts(case):
    """Sizes of a gradient's tensors: spread over the logarithm, none a multiple of anything by design."""
    t, lo, hi = case["tensors"], case["least"], max(case["least"], case["most"])
    return [max(1, int(lo * (hi / lo) ** ((i * 0.6180339887498949) % 1.0))) for i in range(t)]


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype="fp32"):
        return (torch.randn(*shape, generator=gen, device=DEV) * scale).to(DTYPES[dtype])

    def empty(*shape, dtype="fp32"):
        return torch.empty(*shape, device=DEV, dtype=DTYPES[dtype])

    op = case["op"]
    s = {"case": case, "seed": seed}
    if op == "clip":
        kinds = ["bf16" if case["bf16"] and i % 2 else "fp32" for i in range(case["tensors"])]
        s["grads"] = [normal(c, scale=10.0 ** (-(i % 4)), dtype=k) for i, (c, k) in enumerate(zip(_counts(case), kinds))]
        s["out"] = [torch.empty_like(t) for t in s["grads"]]
        s["norm"] = empty(1)
        s["max_norm"] = 1e-2 if case["tight"] else 1e6       # clipped, or let through
        return s
    rows = case["rows"]
    if op in ("norm", "norm8", "norm_grad"):
        w = case["width"]
        s["weight"] = 1.0 + 0.1 * normal(w)
        # hidden features: rows of different sizes, a few columns much larger than the others
        def hidden(dtype):
            t = torch.randn(rows, w, generator=gen, device=DEV)
            t *= torch.exp(torch.randn(rows, 1, generator=gen, device=DEV))
            t[:, :: max(1, w // 4)] *= 8.0
            return t.to(DTYPES[dtype])
        if op == "norm_grad":
            s["h"] = hidden(case["h"])
            s["dy"] = normal(rows, w, scale=1e-3, dtype=case["dy"])
            s["g"] = normal(rows, w, scale=1e-3, dtype=case["h"]) if case["residual"] else None
            s["dh"], s["dweight"] = empty(rows, w, dtype=case["h"]), empty(w)
            return s
        s["x"] = hidden(case["x"])
        s["r"] = normal(rows, w, dtype=case["x"]) if case["residual"] else None
        s["h"] = empty(rows, w, dtype=case["x"]) if case["residual"] else None
        s["y"] = empty(rows, w, dtype=case.get("y", "e4m3"))
        s["scale"] = empty(rows)
        return s
    n, k = case["n"], case["k"]
    if op == "linear":
        c8 = case["dtype"] == "e4m3"
        a, wt = torch.randn(rows, k, generator=gen, device=DEV), torch.randn(n, k, generator=gen, device=DEV) * k ** -0.5
        if c8:
            s["a_scale"], s["w_scale"] = (t.abs().amax(1) / E4M3_MAX for t in (a, wt))
            s["a"], s["w"] = ((t / u[:, None]).to(torch.float8_e4m3fn) for t, u in ((a, s["a_scale"]), (wt, s["w_scale"])))
        else:
            s["a"], s["w"] = a.to(torch.bfloat16), wt.t().contiguous().to(torch.bfloat16)
        s["bias"] = normal(n, scale=0.1)
        s["r"] = normal(rows, n, dtype=case["c"]) if case["residual"] else None
        s["c"] = empty(rows, n, dtype=case["c"])
        s["z"] = empty(rows, n, dtype="bf16") if case["keep"] else None
        return s
    s["dz"] = normal(rows, n, scale=1e-2, dtype="bf16")
    if op == "linear_dx":
        s["w"] = normal(k, n, scale=k ** -0.5, dtype="bf16")
        s["zin"] = normal(rows, k, dtype="bf16") if case["act"] != "none" else None
        s["da"] = empty(rows, k, dtype=case["d"])
        return s
    s["a"] = normal(rows, k, dtype="bf16")
    s["dw"], s["db"] = empty(k, n), empty(n)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "norm8": _own_norm8, "norm_grad": _own_norm_grad, "linear": _own_linear, "linear_dx": _own_linear_dx,
                "linear_dw": _own_linear_dw, "clip": _own_clip}[op](state)
    return {"norm": _norm, "norm8": _norm8, "norm_grad": _norm_grad, "linear": _linear, "linear_dx": _linear_dx, "linear_dw": _linear_dw,
            "clip": _clip}[op](state)


# -- the plain forms
def _rows_normed(s):
    h = s["x"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    return h, h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"]


def _norm(s):
    h, y = _rows_normed(s)
    return {"y": y.to(s["y"].dtype), "h": None if s["r"] is None else h.to(s["x"].dtype)}


def _norm8(s):
    if s["case"]["normalise"]:
        h, y = _rows_normed(s)
    else:
        h = y = s["x"].float()
    scale = (y.abs().amax(1) / E4M3_MAX).clamp_min(TINY_SCALE)
    return {"q": (y / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), "scale": scale,
            "h": None if s["r"] is None else h.to(s["x"].dtype)}


def _norm_grad(s):
    h, dy = s["h"].float(), s["dy"].float()
    rho = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    u = dy * s["weight"]
    dh = rho * u - h * (rho * rho * rho * (u * h).mean(1, keepdim=True))
    if s["g"] is not None:
        dh = dh + s["g"].float()
    return {"dh": dh.to(s["h"].dtype), "dweight": (dy * h * rho).sum(0)}


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return z * 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sg = 1.0 / (1.0 + torch.exp(-z))
    return sg * (1.0 + z * (1.0 - sg))


def _linear(s):
    c = s["case"]
    if c["dtype"] == "e4m3":
        z = (s["a"].float() @ s["w"].float().t()) * s["a_scale"][:, None] * s["w_scale"] + s["bias"]
    else:
        z = s["a"].float() @ s["w"].float() + s["bias"]
    out = _act(z, c["act"])
    if s["r"] is not None:
        out = out + s["r"].float()
    return {"c": out.to(s["c"].dtype), "z": z.to(torch.bfloat16) if c["keep"] else None}


def _linear_dx(s):
    da = s["dz"].float() @ s["w"].float().t()
    if s["zin"] is not None:
        da = da * _act_slope(s["zin"].float(), s["case"]["act"])
    return {"da": da.to(s["da"].dtype)}


def _linear_dw(s):
    dz = s["dz"].float()
    return {"dw": s["a"].float().t() @ dz, "db": dz.sum(0)}


def _clip(s):
    norm = torch.stack([t.double().square().sum() for t in s["grads"]]).sum().sqrt()
    c = torch.where(norm <= s["max_norm"], torch.ones_like(norm), s["max_norm"] / norm).float()
    return {"grads": [(t.float() * c).to(t.dtype) for t in s["grads"]], "norm": norm.float().reshape(1)}


# -- the package's calls
def _code(g, t):
    return {torch.float32: g.DTYPE_FP32, torch.bfloat16: g.DTYPE_BF16, torch.float8_e4m3fn: g.DTYPE_E4M3}[t.dtype]


def _kept(s, nbytes):
    """A workspace of the size that the library asks for, kept from pass to pass."""
    if "workspace" not in s:
        b = nbytes()
        s["workspace"] = torch.empty(b, dtype=torch.uint8, device=DEV) if b else None
    return s["workspace"]


def _own_norm(s):
    import paper_2602_01872_amd as g
    rows, w = s["x"].shape
    g.grp_rmsnorm(rows, w, s["x"], w, _code(g, s["x"]), s["r"], w, s["weight"], EPS, s["h"], w, s["y"], w, _code(g, s["y"]), None)
    return {"y": s["y"], "h": s["h"]}


def _own_norm8(s):
    import paper_2602_01872_amd as g
    rows, w = s["x"].shape
    if s["case"]["normalise"]:
        g.grp_rmsnorm(rows, w, s["x"], w, _code(g, s["x"]), s["r"], w, s["weight"], EPS, s["h"], w, s["y"], w, g.DTYPE_E4M3, s["scale"])
        return {"q": s["y"], "scale": s["scale"], "h": s["h"]}
    g.grp_quantize_rows(rows, w, s["x"], w, _code(g, s["x"]), s["y"], w, s["scale"])
    return {"q": s["y"], "scale": s["scale"], "h": None}


def _own_norm_grad(s):
    import paper_2602_01872_amd as g
    rows, w = s["h"].shape
    ws = _kept(s, lambda: g.grp_rmsnorm_backward_workspace_bytes(rows, w))
    g.grp_rmsnorm_backward(rows, w, s["dy"], w, _code(g, s["dy"]), s["h"], w, _code(g, s["h"]), s["weight"], EPS, s["g"], w, s["dh"], w,
                           s["dweight"], ws)
    return {"dh": s["dh"], "dweight": s["dweight"]}


def _own_linear(s):
    import paper_2602_01872_amd as g
    (m, k), n, c = s["a"].shape, s["c"].shape[1], s["case"]
    ws = _kept(s, lambda: g.grp_linear_workspace_bytes(g.LINEAR_FORWARD, m, n, k, _code(g, s["a"])))
    act = {"none": g.ACT_NONE, "relu": g.ACT_RELU, "gelu": g.ACT_GELU, "silu": g.ACT_SILU}[c["act"]]
    g.grp_linear(m, n, k, s["a"], k, s["w"], s["w"].shape[1], _code(g, s["a"]), s.get("a_scale"), s.get("w_scale"), s["bias"], act,
                 s["r"], n, s["c"], n, _code(g, s["c"]), s["z"], n, ws)
    return {"c": s["c"], "z": s["z"]}


def _own_linear_dx(s):
    import paper_2602_01872_amd as g
    (m, n), k = s["dz"].shape, s["w"].shape[0]
    ws = _kept(s, lambda: g.grp_linear_workspace_bytes(g.LINEAR_DX, m, n, k, g.DTYPE_BF16))
    act = {"none": g.ACT_NONE, "relu": g.ACT_RELU, "gelu": g.ACT_GELU, "silu": g.ACT_SILU}[s["case"]["act"]]
    g.grp_linear_dx(m, n, k, s["dz"], n, s["w"], n, act, s["zin"], k, s["da"], k, _code(g, s["da"]), ws)
    return {"da": s["da"]}


def _own_linear_dw(s):
    import paper_2602_01872_amd as g
    (m, k), n = s["a"].shape, s["dz"].shape[1]
    ws = _kept(s, lambda: g.grp_linear_workspace_bytes(g.LINEAR_DW, m, n, k, g.DTYPE_BF16))
    g.grp_linear_dw(m, n, k, s["a"], k, s["dz"], n, s["dw"], n, s["db"], ws)
    return {"dw": s["dw"], "db": s["db"]}


def _own_clip(s):
    import paper_2602_01872_amd as g
    if "handle" not in s:                # made once for a model's gradients, as a training program does
        s["handle"] = g.grp_gradients_create(s["grads"], s["out"])
    g.grp_clip_gradients(s["handle"], s["max_norm"], s["norm"])
    return {"grads": s["out"], "norm": s["norm"]}


# ------------------------------------------------------------------------------------------------ work
def work(case):
    """Each input read once and each output written once; 2 M N K for a product."""
    op = case["op"]
    if op == "clip":
        cnt = _counts(case)
        el = sum(c * (2 if case["bf16"] and i % 2 else 4) for i, c in enumerate(cnt))
        return {"bytes": 2 * el + 4, "flops": 3 * sum(cnt)}
    m = case["rows"]
    if op in ("norm", "norm8", "norm_grad"):
        w = case["width"]
        if op == "norm_grad":
            h, dy = SIZE[case["h"]], SIZE[case["dy"]]
            return {"bytes": m * w * (dy + h * (3 if case["residual"] else 2)) + 8 * w, "flops": 12 * m * w}
        x = SIZE[case["x"]]
        add = case["residual"]
        out = m * w * SIZE[case["y"]] if op == "norm" else m * (w + 4)
        return {"bytes": m * w * x * (3 if add else 1) + out + (4 * w if case.get("normalise", True) else 0), "flops": 6 * m * w}
    n, k = case["n"], case["k"]
    flops = 2 * m * n * k
    if op == "linear":
        e = SIZE[case["dtype"]]
        b = (m * k + n * k) * e + 4 * n + m * n * (SIZE[case["c"]] * (2 if case["residual"] else 1) + (2 if case["keep"] else 0))
        return {"bytes": b + (4 * (m + n) if e == 1 else 0), "flops": flops}
    if op == "linear_dx":
        return {"bytes": 2 * (m * n + k * n) + m * k * (SIZE[case["d"]] + (2 if case["act"] != "none" else 0)), "flops": flops}
    return {"bytes": 2 * m * (n + k) + 4 * (n * k + n), "flops": flops}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    d = lambda t: None if t is None else t.to(torch.float64)
    if op == "clip":
        flat = torch.cat([d(t) for t in s["grads"]])
        norm = torch.linalg.vector_norm(flat)
        factor = min(1.0, s["max_norm"] / float(norm))
        return {"grads": [v * factor for v in flat.split([t.numel() for t in s["grads"]])], "norm": norm.reshape(1)}
    if op in ("norm", "norm8"):
        h = d(s["x"])
        y = h
        if case.get("normalise", True):
            if s["r"] is not None:
                h = h + d(s["r"])
            y = h / torch.sqrt(h.pow(2).sum(1, keepdim=True) / case["width"] + EPS) * d(s["weight"])
        kept = h if s["r"] is not None else None
        if op == "norm":
            return {"y": y, "h": kept}
        scale = torch.linalg.vector_norm(y, ord=math.inf, dim=1) / E4M3_MAX
        scale = torch.maximum(scale, torch.full_like(scale, TINY_SCALE))
        return {"q": _to_e4m3(y / scale[:, None]), "scale": scale, "h": kept}
    if op == "norm_grad":
        h, dy, wt = d(s["h"]), d(s["dy"]), d(s["weight"])
        size = torch.sqrt(h.pow(2).sum(1, keepdim=True) / case["width"] + EPS)
        unit = h / size                                  # y = unit * weight; d unit / d h = (1 - unit unit^T / width) / size
        back = dy * wt
        dh = (back - unit * ((back * unit).sum(1, keepdim=True) / case["width"])) / size
        if s["g"] is not None:
            dh = dh + d(s["g"])
        return {"dh": dh, "dweight": torch.einsum("ij,ij->j", dy, unit)}
    fn = {"none": lambda z: z, "relu": torch.nn.functional.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}
    if op == "linear":
        if case["dtype"] == "e4m3":
            z = torch.mm(d(s["a"]) * d(s["a_scale"])[:, None], (d(s["w"]) * d(s["w_scale"])[:, None]).t())
        else:
            z = torch.mm(d(s["a"]), d(s["w"]))
        z += d(s["bias"])
        out = fn[case["act"]](z)
        return {"c": out if s["r"] is None else out + d(s["r"]), "z": z if case["keep"] else None}
    if op == "linear_dx":
        da = torch.mm(d(s["dz"]), d(s["w"]).t())
        if s["zin"] is not None:
            zin = d(s["zin"]).requires_grad_()
            fn[case["act"]](zin).backward(da)
            da = zin.grad
        return {"da": da}
    return {"dw": torch.mm(d(s["a"]).t(), d(s["dz"])), "db": d(s["dz"]).sum(0)}


def _to_e4m3(v):
    """Nearest number of 1 + 3 bits of fraction, exponents from -6 on, ties to the even fraction; as 64-bit values."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))).clamp(-6, 8) - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)
