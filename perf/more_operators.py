"""What is measured of a feed-forward block's operators and of its training step: calls as programs make them that train a block or
serve one, from single tokens to the largest batches.

Four operators: the linear layer with bias, activation and residual, the gated pair of linear layers, the norms behind and in front of a
block with its gate and residual scale, each with its gradient, and the norm of many tensors' gradients with their clipping.  A case names
the operator, its sizes and types and what of it is asked for.  Sizes are powers of two and odd numbers between them.
"""
import ctypes
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
MOST_FLOPS, MOST_BYTES = 1.2e12, 1.2e9                      # a drawn case costs no more than the largest listed ones


# ---- cases ---------------------------------------------------------------------------------------------------------

def _gated(name, m, n, k, type="bf16", activation="silu", keep=False, grad=False):
    return dict(name=name, op="gated_grad" if grad else "gated", m=m, n=n, k=k, type=type, activation=activation, keep=keep)


def _linear(name, m, n, k, type="bf16", activation="none", bias=False, residual=False, keep=False, grad=False):
    return dict(name=name, op="linear_grad" if grad else "linear", m=m, n=n, k=k, type=type, activation=activation, bias=bias, residual=residual, keep=keep)


def _norm(name, rows, k, type="bf16", type_r="bf16", post=False, group=0, scale=1.0, grad=False):
    return dict(name=name, op="norm_grad" if grad else "norm", rows=rows, k=k, type=type, type_r=type_r, post=post, group=group, scale=scale)


def _clip(name, layers, k, n, type="bf16", scale=1.0):
    # (16-bit floats' gradients are of a loss times 4096 and stay so)
    return dict(name=name, op="clip", layers=layers, k=k, n=n, type=type, scale=scale, max_norm=4096.0 if type == "f16" else 1.0)


def listed():
    return [
        # serving: one token through the block's two projections, their weights read once
        _gated("gated_1x8192x4096", 1, 8192, 4096),
        # training, forward: the ordinary batch, both projections kept for the gradient
        _gated("gated_4096x8192x4096_keep", 4096, 8192, 4096, keep=True),
        # training, backward: the ordinary batch
        _gated("gated_grad_4096x8192x4096", 4096, 8192, 4096, grad=True),
        # training, backward: odd sizes in every direction, 16-bit floats
        _gated("gated_grad_333x1000x1001", 333, 1000, 1001, type="f16", activation="gelu_tanh", grad=True),
        # serving: one token through the block's last layer, with what the block adds to
        _linear("linear_1x4096x8192_residual", 1, 4096, 8192, residual=True),
        # serving: a batch of 100 sequences, one token each, odd outputs
        _linear("linear_100x5001x2048_bias", 100, 5001, 2048, type="f16", activation="gelu", bias=True),
        # training, backward: a layer with bias and activation
        _linear("linear_grad_4096x8192x2048_bias", 4096, 8192, 2048, activation="gelu_tanh", bias=True, grad=True),
        # serving: one token between two blocks; latency is all of it
        _norm("norm_1x4096", 1, 4096),
        # training, forward: a batch between two blocks, both norms, a gate for each sequence of 1024 tokens, sums in 32 bits
        _norm("norm_8192x4096_post_gate", 8192, 4096, type_r="f32", post=True, group=1024, scale=0.5),
        # training, backward: the same in 16 bits throughout, one gate
        _norm("norm_grad_8192x4096_post_gate", 8192, 4096, post=True, group=8192, scale=0.5, grad=True),
        # training: a small model's gradients in 32 bits, of a loss times 4096
        _clip("clip_2x128x512", 2, 128, 512, type="f32", scale=1.0 / 4096),
        # training: an ordinary model's gradients
        _clip("clip_16x1024x4096", 16, 1024, 4096),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return v | 1 if rng.random() < 0.4 else v if v < 64 else v // 16 * 16

    while True:
        op, type = rng.choice(["gated", "gated_grad", "linear", "linear_grad", "norm", "norm_grad", "clip"]), rng.choice(["bf16", "bf16", "f16"])
        if op.startswith("gated"):
            c = _gated("", size(1, 8192), size(64, 16384), size(64, 8192), type, rng.choice(["silu", "gelu", "gelu_tanh", "relu"]), rng.random() < 0.5,
                       op == "gated_grad")
        elif op.startswith("linear"):
            c = _linear("", size(1, 8192), size(64, 16384), size(64, 16384), type, rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"]),
                        rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.3, op == "linear_grad")
        elif op.startswith("norm"):
            type = rng.choice(["bf16", "bf16", "f16", "f32"])
            rows = size(1, 16384)
            c = _norm("", rows, size(32, 16384), type, rng.choice([type, "f32"]), rng.random() < 0.6, rng.choice([0, rows, size(1, rows)]),
                      rng.choice([1.0, 0.25, 0.7]), op == "norm_grad")
        else:
            k = size(32, 2048)
            c = _clip("", size(1, 48), k, k * rng.randint(1, 4), *rng.choice([("bf16", 1.0), ("f16", 1.0), ("f32", 1.0), ("f32", 1.0 / 4096)]))
        del c["name"]
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


def work(case):
    if case["op"] == "clip":
        n = sum(size * SIZES[type] for size, type in _tensors(case))
        return {"bytes": 2.0 * n, "flops": 3.0 * sum(size for size, _ in _tensors(case))}
    if case["op"].startswith("norm"):
        n, s, sr = case["rows"] * case["k"], SIZES[case["type"]], SIZES[case["type_r"]]
        if case["op"] == "norm":
            return {"bytes": float(n * (2 * s + 2 * sr)), "flops": 8.0 * n}
        return {"bytes": float(n * (3 * s + 3 * sr)), "flops": 20.0 * n}
    m, n, k, s = case["m"], case["n"], case["k"], SIZES[case["type"]]
    if case["op"] == "gated":
        return {"bytes": float(s * (m * k + 2 * n * k + m * n * (3 if case["keep"] else 1))), "flops": 4.0 * m * n * k}
    if case["op"] == "gated_grad":
        return {"bytes": float(s * (2 * m * k + 4 * n * k + 3 * m * n)), "flops": 8.0 * m * n * k}
    if case["op"] == "linear":
        return {"bytes": float(s * (m * k + n * k + m * n * (1 + case["residual"] + case["keep"]))), "flops": 2.0 * m * n * k}
    return {"bytes": float(s * (2 * m * k + 2 * n * k + m * n * (1 + (case["activation"] != "none")))), "flops": 4.0 * m * n * k}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _tensors(case):
    """(elements, type) of a model's parameters: four square and three wide matrices and two 32-bit vectors a layer."""
    k, n = case["k"], case["n"]
    return ([(k * k, case["type"])] * 4 + [(n * k, case["type"])] * 3 + [(k, "f32")] * 2) * case["layers"]


def _padded(rows, k, dtype, fill=None):
    """rows x k with the vectors' starts a multiple of 16 bytes apart."""
    to = 16 // dtype.itemsize
    out = torch.zeros((rows, -(-k // to) * to), dtype=dtype, device="cuda")
    if fill is not None:
        out[:, :k] = fill
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, device="cuda", generator=gen)    # noqa: E731
    state = {"case": case, "ready": False}
    if case["op"] == "clip":
        kinds = _tensors(case)
        state["x"] = []
        for size, type in kinds:
            spread = 1e-4 * case["max_norm"] / case["scale"] * (1.0 + len(state["x"]) % 7)
            state["x"].append(randn(size).mul_(spread).to(TYPES[type]))
        # the clipped gradients lie one behind another, those of a type together
        state["flat"] = {type: torch.zeros((sum(size for size, t in kinds if t == type),), dtype=TYPES[type], device="cuda") for type in dict.fromkeys(t for _, t in kinds)}
        rest = dict(state["flat"])
        state["out"] = []
        for size, type in kinds:
            state["out"].append(rest[type][:size])
            rest[type] = rest[type][size:]
        state["norm"] = torch.zeros((1,), device="cuda")
        # what a program keeps that has its gradients in the same tensors at every step
        state["pointers"] = (ctypes.c_void_p * len(kinds))(*[x.data_ptr() for x in state["x"]])
        state["to"] = (ctypes.c_void_p * len(kinds))(*[x.data_ptr() for x in state["out"]])
        state["sizes"] = (ctypes.c_int64 * len(kinds))(*[size for size, _ in kinds])
        state["types"] = (ctypes.c_int * len(kinds))(*[list(TYPES).index(type) for _, type in kinds])
        return state
    if case["op"].startswith("norm"):
        rows, k, dtype, dtype_r = case["rows"], case["k"], TYPES[case["type"]], TYPES[case["type_r"]]
        loud = torch.where(torch.rand((k,), device="cuda", generator=gen) < 0.01, 20.0, 1.0)
        state["X"] = _padded(rows, k, dtype, randn(rows, k).mul_(loud))
        state["R"] = _padded(rows, k, dtype_r, randn(rows, k).mul_(4.0).mul_(loud))
        state["w_pre"] = 1.0 + 0.1 * randn(k)
        state["w_post"] = 1.0 + 0.1 * randn(k) if case["post"] else None
        state["gate"] = 0.5 * randn(-(-rows // case["group"]), k) if case["group"] else None
        if case["op"] == "norm":
            state["R_out"], state["H"] = _padded(rows, k, dtype_r), _padded(rows, k, dtype)
        else:
            state["dH"], state["dR_out"] = _padded(rows, k, dtype, randn(rows, k)), _padded(rows, k, dtype_r, randn(rows, k))
            state["dX"], state["dR"] = _padded(rows, k, dtype), _padded(rows, k, dtype_r)
            state["dw_pre"] = torch.zeros((k,), device="cuda")
            state["dw_post"] = torch.zeros((k,), device="cuda") if case["post"] else None
            state["dgate"] = torch.zeros_like(state["gate"]) if case["group"] else None
        return state
    m, n, k, dtype = case["m"], case["n"], case["k"], TYPES[case["type"]]
    weights = ["Wg", "Wu"] if case["op"].startswith("gated") else ["W"]
    state["X"] = _padded(m, k, dtype, randn(m, k))
    for w in weights:
        state[w] = _padded(n, k, dtype, randn(n, k).mul_(1.0 / math.sqrt(k)))
    if case["op"].endswith("grad"):
        state["dY"] = _padded(m, n, dtype, randn(m, n).mul_(0.25))
        x = state["X"][:, :k].float()
        bias = 0.1 * randn(n) if case.get("bias") else None
        for w, z in zip(weights, ("G", "U") if len(weights) == 2 else ("Z",)):          # what the forward call left
            v = x @ state[w][:, :k].float().t()
            state[z] = _padded(m, n, dtype, v if bias is None else v + bias)
            state["d" + w] = torch.zeros((n, k), dtype=dtype, device="cuda")
        state["dX"] = torch.zeros((m, k), dtype=dtype, device="cuda")
        if len(weights) == 1:
            state["dbias"] = torch.zeros((n,), device="cuda") if case["bias"] else None
    else:
        outs = ["Y"] + ((["G", "U"] if len(weights) == 2 else ["Z"]) if case["keep"] else [])
        for out in outs:
            state[out] = torch.zeros((m, n), dtype=dtype, device="cuda")
        if len(weights) == 1:
            state["bias"] = (0.1 * randn(n)).to(dtype) if case["bias"] else None
            state["R"] = _padded(m, n, dtype, randn(m, n)) if case["residual"] else None
    return state


# ---- one pass ------------------------------------------------------------------------------------------------------

_kept = {}                                                  # the work memory that a program keeps between its calls


def _library(state):
    """The library with the work memory that the case needs, which a program asks for once."""
    lib = _kept.get("lib")
    if lib is None:
        from paper_2508_00441_amd import binding as lib
        _kept["lib"] = lib
    if not state["ready"]:
        c = state["case"]
        if c["op"] == "clip":
            need = lib.ozaki_gradient_norm_workspace_bytes(len(state["x"]))
        elif c["op"].startswith("norm"):
            need = lib.ozaki_block_norm_workspace_bytes(c["rows"], c["k"], c["group"]) if c["op"] == "norm_grad" else 0
        elif c["op"].startswith("gated"):
            need = lib.ozaki_gated_linear_workspace_bytes(c["m"], c["n"], c["k"], c["op"] == "gated_grad")
        else:
            need = lib.ozaki_linear_workspace_bytes(c["m"], c["n"], c["k"], c["op"] == "linear_grad")
        if _kept.get("ws") is None or _kept["ws"].numel() < need:
            _kept["ws"] = None
            _kept["ws"] = torch.empty(max(need, 1 << 20), dtype=torch.uint8, device="cuda")
            lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
            lib.ozaki_set_workspace(_kept["ws"], _kept["ws"].numel())
        state["ready"] = True
    return lib


def _ld(x):
    return 0 if x is None else x.shape[1]


def _own_pass(state):
    lib, c, s = _library(state), state["case"], state
    if c["op"] == "clip":
        lib.ozaki_clip_gradients(len(s["x"]), s["pointers"], s["sizes"], s["types"], c["scale"], c["max_norm"], s["to"], s["norm"])
        return {"norm": s["norm"]} | s["flat"]
    type = lib.TYPES[c["type"]]
    if c["op"].startswith("norm"):
        rows, k, type_r = c["rows"], c["k"], lib.TYPES[c["type_r"]]
        a = (rows, k, s["X"], _ld(s["X"]), type, s["w_post"], s["gate"], c["group"], c["scale"], EPS)
        if c["op"] == "norm":
            lib.ozaki_block_norm(*a, s["R"], _ld(s["R"]), type_r, s["R_out"], _ld(s["R_out"]), s["w_pre"], s["H"], _ld(s["H"]))
            return {"r": s["R_out"][:, :k], "h": s["H"][:, :k]}
        lib.ozaki_block_norm_grad(*a, s["R"], _ld(s["R"]), type_r, s["w_pre"], s["dH"], _ld(s["dH"]), s["dR_out"], _ld(s["dR_out"]), s["dX"], _ld(s["dX"]),
                                  s["dR"], _ld(s["dR"]), s["dw_post"], s["dgate"], s["dw_pre"])
        out = {"dx": s["dX"][:, :k], "dr": s["dR"][:, :k], "dw_pre": s["dw_pre"]}
        return out | ({"dw_post": s["dw_post"]} if c["post"] else {}) | ({"dgate": s["dgate"]} if c["group"] else {})
    m, n, k, activation = c["m"], c["n"], c["k"], lib.ACTIVATIONS[c["activation"]]
    if c["op"] == "gated":
        G, U = s.get("G"), s.get("U")
        lib.ozaki_gated_linear(m, n, k, s["X"], _ld(s["X"]), s["Wg"], s["Wu"], _ld(s["Wg"]), type, activation, s["Y"], n, G, _ld(G), U, _ld(U))
        return {"y": s["Y"]} | ({"g": G, "u": U} if c["keep"] else {})
    if c["op"] == "gated_grad":
        lib.ozaki_gated_linear_grad(m, n, k, s["X"], _ld(s["X"]), s["Wg"], s["Wu"], _ld(s["Wg"]), type, activation, s["G"], _ld(s["G"]), s["U"], _ld(s["U"]),
                                    s["dY"], _ld(s["dY"]), s["dX"], k, s["dWg"], s["dWu"], k)
        return {"dx": s["dX"], "dwg": s["dWg"], "dwu": s["dWu"]}
    if c["op"] == "linear":
        Z = s.get("Z")
        lib.ozaki_linear(m, n, k, s["X"], _ld(s["X"]), s["W"], _ld(s["W"]), type, s["bias"], activation, s["R"], _ld(s["R"]), s["Y"], n, Z, _ld(Z))
        return {"y": s["Y"]} | ({"z": Z} if c["keep"] else {})
    lib.ozaki_linear_grad(m, n, k, s["X"], _ld(s["X"]), s["W"], _ld(s["W"]), type, activation, s["Z"], _ld(s["Z"]), s["dY"], _ld(s["dY"]), s["dX"], k,
                          s["dW"], k, s["dbias"])
    return {"dx": s["dX"], "dw": s["dW"]} | ({"dbias": s["dbias"]} if c["bias"] else {})


# ---- the plain form --------------------------------------------------------------------------------------------------

def _activated(z, activation):
    """The activation's value and derivative."""
    if activation == "none":
        return z, torch.ones_like(z)
    if activation == "relu":
        return z.clamp(min=0.0), (z > 0).to(z.dtype)
    if activation == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return z * p, p * (1.0 + z * (1.0 - p))
    if activation == "gelu":
        p = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * p, p + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)


def _spread_gate(gate, group, rows):
    return gate[torch.arange(rows, device="cuda") // group]


def _plain_norm(state):
    c, s = state["case"], state
    rows, k, dtype, dtype_r = c["rows"], c["k"], TYPES[c["type"]], TYPES[c["type_r"]]
    x, r = s["X"][:, :k].float(), s["R"][:, :k].float()
    gate = c["scale"] * _spread_gate(s["gate"], c["group"], rows) if c["group"] else c["scale"]
    rho = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) if c["post"] else None
    if c["op"] == "norm":
        r = r + gate * (x * rho * s["w_post"] if c["post"] else x)
        h = r * torch.rsqrt((r * r).mean(1, keepdim=True) + EPS) * s["w_pre"]
        return {"r": r.to(dtype_r), "h": h.to(dtype)}
    dh = s["dH"][:, :k].float()
    rho_r = torch.rsqrt((r * r).mean(1, keepdim=True) + EPS)
    normed, dn = r * rho_r, dh * s["w_pre"]
    dr = s["dR_out"][:, :k].float() + rho_r * (dn - normed * (dn * normed).mean(1, keepdim=True))
    out = {"dr": dr.to(dtype_r), "dw_pre": (dh * normed).sum(0)}
    if c["post"]:
        m, dm = x * rho, gate * dr * s["w_post"]
        out["dx"] = (rho * (dm - m * (dm * m).mean(1, keepdim=True))).to(dtype)
        out["dw_post"] = (gate * dr * m).sum(0)
        u = m * s["w_post"]
    else:
        out["dx"], u = (gate * dr).to(dtype), x
    if c["group"]:
        per_row = c["scale"] * dr * u
        groups = torch.arange(rows, device="cuda") // c["group"]
        out["dgate"] = torch.zeros_like(s["gate"]).index_add_(0, groups, per_row)
    return out


def run(state):
    if own:
        return _own_pass(state)
    c, s = state["case"], state
    if c["op"] == "clip":
        total = torch.stack([x.double().square().sum() for x in s["x"]]).sum()
        norm = (c["scale"] * total.sqrt()).float().reshape(1)
        factor = c["scale"] * (c["max_norm"] / norm).clamp(max=1.0)
        _ = [to.copy_(x.float() * factor) for x, to in zip(s["x"], s["out"])]
        return {"norm": norm} | s["flat"]
    if c["op"].startswith("norm"):
        return _plain_norm(state)
    m, n, k, dtype = c["m"], c["n"], c["k"], TYPES[c["type"]]
    x = s["X"][:, :k].float()
    if c["op"] == "gated":
        g, u = (x @ s[w][:, :k].float().t() for w in ("Wg", "Wu"))
        return {"y": (_activated(g, c["activation"])[0] * u).to(dtype)} | ({"g": g.to(dtype), "u": u.to(dtype)} if c["keep"] else {})
    if c["op"] == "linear":
        z = x @ s["W"][:, :k].float().t()
        if c["bias"]:
            z = z + s["bias"].float()
        y = _activated(z, c["activation"])[0]
        if c["residual"]:
            y = y + s["R"][:, :n].float()
        return {"y": y.to(dtype)} | ({"z": z.to(dtype)} if c["keep"] else {})
    dy = s["dY"][:, :n].float()
    if c["op"] == "gated_grad":
        u, (a, slope) = s["U"][:, :n].float(), _activated(s["G"][:, :n].float(), c["activation"])
        dg, du = dy * u * slope, dy * a
        dx = dg @ s["Wg"][:, :k].float() + du @ s["Wu"][:, :k].float()
        return {"dx": dx.to(dtype), "dwg": (dg.t() @ x).to(dtype), "dwu": (du.t() @ x).to(dtype)}
    dz = dy * _activated(s["Z"][:, :n].float(), c["activation"])[1]
    out = {"dx": (dz @ s["W"][:, :k].float()).to(dtype), "dw": (dz.t() @ x).to(dtype)}
    return out | ({"dbias": dz.sum(0)} if c["bias"] else {})


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _value(z, activation):
    if activation == "none":
        return z
    if activation == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if activation == "silu":
        return z * torch.sigmoid(z)
    if activation == "gelu":
        return z * torch.special.ndtr(z)
    return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))     # (1 + tanh y) / 2 = sigmoid 2y


def _slope(z, activation):
    with torch.enable_grad():
        z = z.clone().requires_grad_()
        return torch.autograd.grad(_value(z, activation).sum(), z)[0] if activation != "none" else torch.ones_like(z)


def _exact_norm(c, s):
    rows, k = c["rows"], c["k"]
    leaves = {name: s[name].double().requires_grad_() for name in ("w_pre", "w_post", "gate") if s[name] is not None}
    out = {"r": [], "h": [], "dx": [], "dr": []}

    def normed(v, w):
        return v / torch.sqrt(v.square().sum(1, keepdim=True) / k + EPS) * w

    for at in range(0, rows, 4096):                         # some rows at a time
        part = slice(at, min(rows, at + 4096))
        x, r = (s[name][part, :k].double().requires_grad_() for name in ("X", "R"))
        added = normed(x, leaves["w_post"]) if c["post"] else x
        if c["group"]:
            added = added * leaves["gate"][torch.arange(part.start, part.stop, device="cuda") // c["group"]]
        if c["op"] == "norm":
            total = r + c["scale"] * added
            out["r"].append(total.detach())
            out["h"].append(normed(total, leaves["w_pre"]).detach())
            continue
        # r is the sum that the forward call left: its own gradient first, then that of what was added
        (normed(r, leaves["w_pre"]) * s["dH"][part, :k].double()).sum().backward()
        dr = r.grad + s["dR_out"][part, :k].double()
        (c["scale"] * added * dr).sum().backward()
        out["dr"].append(dr)
        out["dx"].append(x.grad)
    out = {name: torch.cat(parts) for name, parts in out.items() if parts}
    return out if c["op"] == "norm" else out | {"d" + name: leaf.grad for name, leaf in leaves.items()}


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "clip":
        norm = c["scale"] * math.sqrt(math.fsum(float(x.double().norm()) ** 2 for x in s["x"]))
        factor = c["scale"] * min(1.0, c["max_norm"] / norm)
        return {"norm": torch.tensor([norm], dtype=torch.float64)} | {type: torch.cat([x.double() * factor for x in s["x"] if x.dtype == TYPES[type]])
                                                                      for type in s["flat"]}
    if c["op"].startswith("norm"):
        return _exact_norm(c, s)
    n, k, activation = c["n"], c["k"], c["activation"]
    wide = lambda name, width: s[name][:, :width].double()    # noqa: E731
    x = wide("X", k)
    if c["op"] == "gated":
        g, u = torch.mm(x, wide("Wg", k).t()), torch.mm(x, wide("Wu", k).t())
        return {"y": _value(g, activation) * u} | ({"g": g, "u": u} if c["keep"] else {})
    if c["op"] == "linear":
        z = torch.mm(x, wide("W", k).t()) + (s["bias"].double() if c["bias"] else 0.0)
        return {"y": _value(z, activation) + (wide("R", n) if c["residual"] else 0.0)} | ({"z": z} if c["keep"] else {})
    dy = wide("dY", n)
    if c["op"] == "gated_grad":
        dg, du = dy * wide("U", n) * _slope(wide("G", n), activation), dy * _value(wide("G", n), activation)
        return {"dx": torch.mm(dg, wide("Wg", k)) + torch.mm(du, wide("Wu", k)), "dwg": torch.mm(dg.t(), x), "dwu": torch.mm(du.t(), x)}
    dz = dy * _slope(wide("Z", n), activation)
    return {"dx": torch.mm(dz, wide("W", k)), "dw": torch.mm(dz.t(), x)} | ({"dbias": dz.sum(0)} if c["bias"] else {})
