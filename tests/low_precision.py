"""Plain 64-bit forms of the low-precision operators and the operands that their tests share."""
import torch

BLOCK = 128
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
#: half a unit in the last place over the smallest number of a binade (24, 8 and 11 significant bits), and half of the smallest step
ROUNDING = {"f32": (2.0 ** -24, 2.0 ** -150), "bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25)}


def ceil(n, to):
    return -(-n // to) * to


def padded(x, to, fill):
    """x (rows x k) with vectors that start a multiple of `to` elements apart; `fill` behind their ends."""
    out = torch.full((x.shape[0], ceil(x.shape[1], to) + to), fill, dtype=x.dtype)
    out[:, : x.shape[1]] = x
    return out


def block_amax(x, blocks):
    """[k block, row or row block] of the finite magnitudes of a CPU tensor, at least 2^-100."""
    rows, k = x.shape
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    out = []
    for e in range(0, k, BLOCK):
        row = a[:, e: e + BLOCK].amax(1)
        out.append(torch.stack([row[r: r + BLOCK].amax() for r in range(0, rows, BLOCK)]) if blocks else row)
    return torch.stack(out).clamp(min=2.0 ** -100)


def spread(s, rows, k, blocks):
    """[k block, row (block)] -> rows x k."""
    s = s.t()
    if blocks:
        s = s.repeat_interleave(BLOCK, 0)[:rows]
    return s.repeat_interleave(BLOCK, 1)[:, :k]


def to_e4m3(y):
    """The nearest E4M3 value of 64-bit numbers up to 448 in magnitude, ties to even: steps of 2^-3 of the binade, of 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(y / step) * step).float().to(torch.float8_e4m3fn)


def quantised(x, blocks):
    """Codes (float8_e4m3fn) and scales of a CPU float32 tensor: the quotient in 64 bits (its numerator is exact, so that ties are ties)."""
    amax = block_amax(x, blocks)
    y = x.double() * 448.0 / spread(amax.double(), x.shape[0], x.shape[1], blocks)
    return to_e4m3(torch.where(torch.isfinite(y), y, torch.full_like(y, float("nan")))), amax / torch.full_like(amax, 448.0)


def dequantised(q, s, blocks):
    return q.double() * spread(s.double(), q.shape[0], q.shape[1], blocks)


def cut_products(q, s, blocks):
    """For groups of eight neighbouring codes the power of two of the largest exponent times the scale: rows x groups."""
    x = torch.nn.functional.pad(q.float().abs(), (0, -q.shape[1] % 8)).reshape(q.shape[0], -1, 8).amax(2).double()
    e = torch.floor(torch.log2(x.clamp(min=2.0 ** -6)))
    return torch.exp2(e) * spread(s.double(), q.shape[0], q.shape[1], blocks)[:, ::8]


def gemm_bound(k, magnitudes, type_d, result, cut):
    """What D may be off: the matrix unit's 128 additions of a block, each allowed twice a rounding; a rounding for the scales' product and one
    for each block's multiply-add; D's own rounding.  A D of 16 bits takes the FP8 instructions, which cut each of eight neighbouring products at 2^-13 of the
    largest's power of two (`cut`: the sum of those, times the scales); a D of 32 bits takes others."""
    rel, tiny = ROUNDING[type_d]
    off = (2 * BLOCK + ceil(k, BLOCK) // BLOCK + 4) * 2.0 ** -24 * magnitudes + (0.0 if type_d == "f32" else 8 * 2.0 ** -13 * cut)
    return off * (1 + rel) + rel * result.abs() + tiny


def loss_forward(h, w, targets, ignore):
    """loss, lse, logits in 64 bits."""
    z = h.double() @ w.double().t()
    lse = torch.logsumexp(z, 1)
    counts = targets != ignore
    picked = z.gather(1, targets.clamp(0, w.shape[0] - 1).unsqueeze(1)).squeeze(1)
    return torch.where(counts, lse - picked, torch.zeros_like(lse)), lse, z


def loss_gradient(h, w, targets, ignore, lse, dloss):
    """dH, dW and g in 64 bits; tokens that do not count have no share, whatever their rows of h hold."""
    counts = targets != ignore
    h = torch.where(counts.unsqueeze(1), h.double(), 0.0)
    z = h @ w.double().t()
    p = torch.exp(z - lse.double().unsqueeze(1))
    g = p.clone()
    g[torch.arange(len(targets)), targets.clamp(0, w.shape[0] - 1)] -= 1.0
    factor = torch.where(counts, dloss.double(), 0.0).unsqueeze(1)
    g = torch.where(counts.unsqueeze(1), g * factor, 0.0)
    p = torch.where(counts.unsqueeze(1), p * factor.abs(), 0.0)
    return g @ w.double(), g.t() @ h, g, p, h


def logit_error(h, w):
    """What a token's z may be off: k additions, each allowed twice a rounding."""
    return 2 * (h.shape[1] + 2) * 2.0 ** -24 * (h.double().abs() @ w.double().abs().t()).amax(1)
