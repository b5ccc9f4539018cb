"""What is measured of the low-precision operators: calls as programs make them that train a layer or a language model's output
layer, or that serve one, from single tokens to the largest batches.

Three operators: the quantisation of a matrix to 8-bit floating point (OCP E4M3) with a scale for each block of 128, the product of
two matrices in that form, and the softmax cross entropy of a linear layer's outputs over a vocabulary, with its gradient.  A
case names the operator, its sizes, the types and where scales lie.  Sizes are powers of two and odd numbers between them.
"""
import math

import torch

own = False

BLOCK = 128                                                 # elements that share a scale, along one axis or both
E4M3_MAX = 448.0
SMALLEST_AMAX = 2.0 ** -100                                 # what a block of smaller values is scaled by
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
MOST_FLOPS, MOST_BYTES = 6.5e12, 1.6e9                      # a drawn case costs no more than the largest listed ones


# ---- cases ---------------------------------------------------------------------------------------------------------

def _quantise(name, rows, k, type, blocks=False, both=False):
    return dict(name=name, op="quantise", rows=rows, k=k, type=type, blocks=blocks, both=both)


def _gemm(name, m, n, k, blocks=True, type="bf16"):
    return dict(name=name, op="gemm", m=m, n=n, k=k, blocks=blocks, type=type)


def _loss(name, tokens, vocab, k, grad, type="bf16", ignored=0.0):
    return dict(name=name, op="loss_grad" if grad else "loss", tokens=tokens, vocab=vocab, k=k, type=type, ignored=ignored)


def listed():
    return [
        # serving: one token's activations before an 8-bit product; latency is all of it
        _quantise("quantise_1x4096", 1, 4096, "bf16"),
        # training: a batch's activations, along the features for the layer's product and along the tokens for the weight's gradient
        _quantise("quantise_8192x4096_both", 8192, 4096, "bf16", both=True),
        # after an optimizer step: the 32-bit weights, in squares, as they are and transposed for the input's gradient
        _quantise("quantise_weights_16384x4096", 16384, 4096, "f32", blocks=True, both=True),
        # serving: one token through a layer, the weights read once
        _gemm("gemm_1x8192x4096", 1, 8192, 4096),
        # serving: a batch of 64 sequences, one token each, a long inner dimension and few outputs
        _gemm("gemm_64x4096x16384", 64, 4096, 16384),
        # odd sizes in every direction, a short prompt
        _gemm("gemm_333x1000x1301", 333, 1000, 1301, type="f32"),
        # training, forward: the ordinary size
        _gemm("gemm_4096x4096x4096", 4096, 4096, 4096),
        # training, the weight's gradient: both operands scaled along the tokens, 32-bit result
        _gemm("gemm_16384x4096x8192_vectors", 16384, 4096, 8192, blocks=False, type="f32"),
        # scoring an answer of a few tokens: the vocabulary's weights read once
        _loss("loss_16x65536x2048", 16, 65536, 2048, False),
        # evaluation: a batch of prompts, the largest vocabulary
        _loss("loss_4096x131072x4096", 4096, 131072, 4096, False),
        # training on answers only, odd sizes everywhere
        _loss("grad_1003x50001x1000_ignored", 1003, 50001, 1000, True, type="f16", ignored=0.6),
        # training: the ordinary batch
        _loss("grad_4096x65536x4096", 4096, 65536, 4096, True),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return v | 1 if rng.random() < 0.4 else v if v < 64 else v // 16 * 16

    while True:
        op = rng.choice(["quantise", "gemm", "gemm", "loss", "loss_grad"])
        if op == "quantise":
            blocks = rng.random() < 0.4
            c = _quantise("", size(1, 16384), size(64, 16384), rng.choice(["bf16", "bf16", "f16", "f32"]), blocks, rng.random() < 0.5)
        elif op == "gemm":
            c = _gemm("", size(1, 16384), size(128, 16384), size(128, 16384), rng.random() < 0.6, rng.choice(["bf16", "bf16", "f16", "f32"]))
        else:
            c = _loss("", size(1, 8192), size(1000, 131072), size(64, 8192), op == "loss_grad", rng.choice(["bf16", "bf16", "f16"]),
                      rng.choice([0.0, 0.0, 0.1, 0.6]))
        del c["name"]
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


def work(case):
    if case["op"] == "quantise":
        n = case["rows"] * case["k"]
        copies = 2 if case["both"] else 1
        scales = 4.0 * copies * n / (BLOCK * BLOCK if case["blocks"] else BLOCK)
        return {"bytes": float(n * (SIZES[case["type"]] + copies)) + scales, "flops": 4.0 * n}
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        scales = 4.0 * k / BLOCK * (m + (n / BLOCK if case["blocks"] else n))
        return {"bytes": float(m * k + n * k + m * n * SIZES[case["type"]]) + scales, "flops": 2.0 * m * n * k}
    t, v, k, size = case["tokens"], case["vocab"], case["k"], SIZES[case["type"]]
    if case["op"] == "loss":
        return {"bytes": float(size * (t + v) * k + 16 * t), "flops": 2.0 * t * v * k}
    # the logits again, and the two gradients
    return {"bytes": float(size * (2 * t + 2 * v) * k + 16 * t), "flops": 6.0 * t * v * k}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _ceil(n, to):
    return -(-n // to) * to


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _padded(rows, k, dtype, to):
    """rows x k with the vectors' starts a multiple of `to` elements apart."""
    return torch.zeros((rows, _ceil(k, to)), dtype=dtype, device="cuda")


def _activations(rows, k, gen):
    """Normally distributed, a few features a good deal larger than the others."""
    x = torch.randn((rows, k), device="cuda", generator=gen)
    loud = torch.rand((k,), device="cuda", generator=gen) < 0.01
    return x.mul_(torch.where(loud, 20.0, 1.0))


def _in_blocks(x):
    """Rows x k with the rows and k filled up to whole blocks: [row block, 128, k block, 128]."""
    r, k = x.shape
    rp, kp = _ceil(r, BLOCK), _ceil(k, BLOCK)
    y = torch.zeros((rp, kp), dtype=x.dtype, device=x.device)
    y[:r, :k] = x
    return y.view(rp // BLOCK, BLOCK, kp // BLOCK, BLOCK)


def _plain_scales(x, blocks):
    """The largest finite magnitude of each block of the rows' elements (blocks: of each square), [k block, row (block)]."""
    y = _in_blocks(torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)))
    amax = y.amax(dim=(1, 3)) if blocks else y.amax(dim=3).reshape(-1, y.shape[2])[: x.shape[0]]
    return amax.clamp(min=SMALLEST_AMAX).t().contiguous()


def _spread(s, rows, k, blocks):
    """[k block, row (block)] -> rows x k."""
    s = s.t()
    if blocks:
        s = s.repeat_interleave(BLOCK, 0)[:rows]
    return s.repeat_interleave(BLOCK, 1)[:, :k]


def _plain_quantise(x, blocks):
    amax = _plain_scales(x, blocks)
    q = (x * _spread(E4M3_MAX / amax, x.shape[0], x.shape[1], blocks)).to(torch.float8_e4m3fn)
    return q, amax / E4M3_MAX


def _quantised(x, blocks):
    """An operand of a product as a program has it in hand: the bytes with padded vectors, and the scales."""
    q, s = _plain_quantise(x, blocks)
    to = _padded(x.shape[0], x.shape[1], torch.uint8, 16)
    to[:, : x.shape[1]] = q.view(torch.uint8)
    return to, s


def prepare(case, seed):
    gen = _generator(seed)
    state = {"case": case, "ready": False}
    if case["op"] == "quantise":
        rows, k, to = case["rows"], case["k"], 16 // SIZES[case["type"]]
        x = torch.randn((rows, k), device="cuda", generator=gen).mul_(0.02) if case["blocks"] else _activations(rows, k, gen)
        X = _padded(rows, k, TYPES[case["type"]], to)
        X[:, :k] = x
        state["X"] = X
        blocked = lambda n: -(-n // BLOCK) if case["blocks"] else n    # noqa: E731
        state["Q"], state["S"] = _padded(rows, k, torch.uint8, 16), torch.zeros((-(-k // BLOCK), blocked(rows)), device="cuda")
        if case["both"]:
            state["Qt"], state["St"] = _padded(k, rows, torch.uint8, 16), torch.zeros((-(-rows // BLOCK), blocked(k)), device="cuda")
    elif case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        state["A"], state["SA"] = _quantised(_activations(m, k, gen), False)
        state["B"], state["SB"] = _quantised(torch.randn((n, k), device="cuda", generator=gen).mul_(0.02), case["blocks"])
        state["D"] = torch.zeros((m, n), dtype=TYPES[case["type"]], device="cuda")
    else:
        t, v, k, dtype = case["tokens"], case["vocab"], case["k"], TYPES[case["type"]]
        H, W = _padded(t, k, dtype, 8), _padded(v, k, dtype, 8)
        H[:, :k] = torch.randn((t, k), device="cuda", generator=gen)
        W[:, :k] = torch.randn((v, k), device="cuda", generator=gen).mul_(2.0 / math.sqrt(k))
        targets = torch.randint(0, v, (t,), device="cuda", generator=gen)
        targets[torch.rand((t,), device="cuda", generator=gen) < case["ignored"]] = -100
        state |= {"H": H, "W": W, "targets": targets}
        state["loss"], state["lse"] = torch.zeros((t,), device="cuda"), torch.zeros((t,), device="cuda")
        if case["op"] == "loss_grad":
            # what the forward call left, and the mean's gradient (16-bit floats: of the loss times a scale, as such training needs it)
            state["lse"] = torch.cat([torch.logsumexp(part[:, :k].float() @ W[:, :k].float().t(), 1) for part in H.split(1024)])
            state["dloss"] = torch.full((t,), (4096.0 if case["type"] == "f16" else 1.0) / max(1, int((targets >= 0).sum())), device="cuda")
            state["dH"] = torch.zeros((t, k), dtype=dtype, device="cuda")
            state["dW"] = torch.zeros((v, k), dtype=dtype, device="cuda")
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
        need = 256
        if c["op"] == "gemm":
            need = lib.ozaki_gemm_fp8_workspace_bytes(c["m"], c["n"], c["k"])
        elif c["op"] != "quantise":
            need = lib.ozaki_linear_loss_workspace_bytes(c["tokens"], c["vocab"], c["k"], c["op"] == "loss_grad", False)
        if _kept.get("ws") is None or _kept["ws"].numel() < need:
            _kept["ws"] = None
            _kept["ws"] = torch.empty(max(need, 1 << 20), dtype=torch.uint8, device="cuda")
            lib.ozaki_set_stream(torch.cuda.current_stream().cuda_stream)
            lib.ozaki_set_workspace(_kept["ws"], _kept["ws"].numel())
        state["ready"] = True
    return lib


def _own_pass(state):
    lib, c = _library(state), state["case"]
    if c["op"] == "quantise":
        X, Q, S, Qt, St = state["X"], state["Q"], state["S"], state.get("Qt"), state.get("St")
        lib.ozaki_quantise_fp8(c["rows"], c["k"], X, X.shape[1], lib.TYPES[c["type"]], lib.SCALE_BLOCKS if c["blocks"] else lib.SCALE_VECTORS,
                               Q, Q.shape[1], S, S.shape[1], Qt, Qt.shape[1] if c["both"] else 0, St, St.shape[1] if c["both"] else 0)
        out = {"q": Q[:, : c["k"]].view(torch.float8_e4m3fn), "s": S}
        if c["both"]:
            out |= {"qt": Qt[:, : c["rows"]].view(torch.float8_e4m3fn), "st": St}
        return out
    if c["op"] == "gemm":
        A, B, D = state["A"], state["B"], state["D"]
        lib.ozaki_gemm_fp8(c["m"], c["n"], c["k"], A, A.shape[1], state["SA"], c["m"], B, B.shape[1], state["SB"], state["SB"].shape[1],
                           lib.SCALE_BLOCKS if c["blocks"] else lib.SCALE_VECTORS, D, c["n"], lib.TYPES[c["type"]])
        return D
    H, W = state["H"], state["W"]
    a = (c["tokens"], c["vocab"], c["k"], H, H.shape[1], W, W.shape[1], lib.TYPES[c["type"]], state["targets"], -100)
    if c["op"] == "loss":
        lib.ozaki_linear_loss(*a, state["loss"], state["lse"])
        return {"loss": state["loss"], "lse": state["lse"]}
    lib.ozaki_linear_loss_grad(*a, state["lse"], state["dloss"], state["dH"], c["k"], state["dW"], c["k"])
    return {"dh": state["dH"], "dw": state["dW"]}


def run(state):
    if own:
        return _own_pass(state)
    c = state["case"]
    if c["op"] == "quantise":
        x = state["X"][:, : c["k"]].float()
        out = dict(zip(("q", "s"), _plain_quantise(x, c["blocks"])))
        if c["both"]:
            out |= dict(zip(("qt", "st"), _plain_quantise(x.t(), c["blocks"])))
        return out
    if c["op"] == "gemm":
        m, n, k = c["m"], c["n"], c["k"]
        a = state["A"][:, :k].view(torch.float8_e4m3fn).float() * _spread(state["SA"], m, k, False)
        b = state["B"][:, :k].view(torch.float8_e4m3fn).float() * _spread(state["SB"], n, k, c["blocks"])
        return (a @ b.t()).to(TYPES[c["type"]])
    k, targets = c["k"], state["targets"]
    h, w = state["H"][:, :k].float(), state["W"][:, :k].float()
    valid, at = targets >= 0, targets.clamp(min=0).unsqueeze(1)
    logits = h @ w.t()
    if c["op"] == "loss":
        most = logits.amax(1, keepdim=True)
        lse = (logits - most).exp().sum(1, keepdim=True).log() + most
        loss = torch.where(valid, (lse - logits.gather(1, at)).squeeze(1), 0.0)
        return {"loss": loss, "lse": lse.squeeze(1)}
    g = logits.sub_(state["lse"].unsqueeze(1)).exp_()
    g.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
    g.mul_(torch.where(valid, state["dloss"], 0.0).unsqueeze(1))
    return {"dh": (g @ w).to(state["dH"].dtype), "dw": (g.t() @ h).to(state["dW"].dtype)}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _to_e4m3(y):
    """The nearest value of E4M3, ties to the even significand: multiples of 2^-3 of the binade, of 2^-9 below 2^-6."""
    _, e = torch.frexp(y.abs().clamp(min=2.0 ** -6))
    step = torch.pow(2.0, (e - 4).double())
    return (torch.round(y / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_quantise(x, blocks):
    rows, k = x.shape
    r, e = torch.arange(rows, device="cuda") // (BLOCK if blocks else 1), torch.arange(k, device="cuda") // BLOCK
    amax = torch.zeros((int(e[-1]) + 1, rows), dtype=torch.float64, device="cuda")
    amax = amax.scatter_reduce(0, e.unsqueeze(1).expand(k, rows), x.abs().t(), "amax")
    if blocks:
        squares = torch.zeros((amax.shape[0], int(r[-1]) + 1), dtype=torch.float64, device="cuda")
        amax = squares.scatter_reduce(1, r.unsqueeze(0).expand(amax.shape), amax, "amax")
    amax = amax.clamp(min=SMALLEST_AMAX)
    each = amax[e][:, r].t()
    return _to_e4m3(x * (E4M3_MAX / each)), amax / E4M3_MAX


def exact(case, seed):
    state, c = prepare(case, seed), case
    if c["op"] == "quantise":
        x = state["X"][:, : c["k"]].double()
        q, s = _exact_quantise(x, c["blocks"])
        out = {"q": q, "s": s}
        if c["both"]:
            out["qt"], out["st"] = _exact_quantise(x.t().contiguous(), c["blocks"])
        return out
    if c["op"] == "gemm":
        m, n, k = c["m"], c["n"], c["k"]
        total = torch.zeros((m, n), dtype=torch.float64, device="cuda")
        for kb in range(-(-k // BLOCK)):                    # block by block, as the definition says
            at = slice(kb * BLOCK, min(k, (kb + 1) * BLOCK))
            a, b = (state[o][:, at].contiguous().view(torch.float8_e4m3fn).double() for o in ("A", "B"))
            sb = state["SB"][kb].double()
            if c["blocks"]:
                sb = sb[torch.arange(n, device="cuda") // BLOCK]
            total += (a * state["SA"][kb].double().unsqueeze(1)) @ (b * sb.unsqueeze(1)).t()
        return total
    k, targets = c["k"], state["targets"]
    H, W = state["H"][:, :k].double(), state["W"][:, :k].double()
    outs = {"loss": [], "lse": [], "dh": []}
    dw = torch.zeros_like(W) if c["op"] == "loss_grad" else None
    for t0 in range(0, c["tokens"], 1024):                  # the logits of some tokens at a time
        h, y = H[t0: t0 + 1024], targets[t0: t0 + 1024]
        logits = torch.mm(h, W.t())
        valid, rows = y >= 0, torch.arange(len(y), device="cuda")
        if c["op"] == "loss":
            lse = torch.logsumexp(logits, 1)
            outs["lse"].append(lse)
            outs["loss"].append(torch.where(valid, lse - logits[rows, y.clamp(min=0)], 0.0))
            continue
        p = torch.exp(logits - state["lse"][t0: t0 + 1024].double().unsqueeze(1))
        p[rows[valid], y[valid]] -= 1.0
        p *= torch.where(valid, state["dloss"][t0: t0 + 1024].double(), 0.0).unsqueeze(1)
        outs["dh"].append(torch.mm(p, W))
        dw += torch.mm(p.t(), h)
    if c["op"] == "loss":
        return {"loss": torch.cat(outs["loss"]), "lse": torch.cat(outs["lse"])}
    return {"dh": torch.cat(outs["dh"]), "dw": dw}
