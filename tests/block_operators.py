"""Plain 64-bit forms of the feed-forward block's operators with what their 32-bit evaluation may be off, for tensors on any device."""
import math

import torch

from low_precision import DTYPES, ROUNDING

ULP = 2.0 ** -24                                                    # half a unit in the last place, relative, of 24 bits
TINY = 2.0 ** -126


def stored(x, type):
    """What rounding a number of x's magnitude to the type may change."""
    rel, tiny = ROUNDING[type]
    return rel * x.abs() + tiny


def rounded(want, off, type):
    """What a result may be off that is `off` away from `want` before it is rounded to the type."""
    return off + stored(want.abs() + off, type)


def padded(x, type, fill=float("nan"), more=0):
    """x (rows x k) on the GPU with vectors that start a multiple of 16 bytes apart, `fill` behind their ends."""
    dtype = DTYPES[type]
    to = 16 // dtype.itemsize
    out = torch.full((x.shape[0], -(-x.shape[1] // to) * to + more * to), fill, dtype=dtype, device="cuda")
    out[:, : x.shape[1]] = x
    return out


def activation(z, name):
    """The activation's value and derivative, and what 32 bits may be off of each.

    The sigmoid of a: the exponential's argument is off by a few roundings of |a|, which its relative error is, the quotient by a few of its own (16 in all
    with the products around it).  Phi of z: an error of two roundings in z / sqrt(2) changes erfc by 2 z^2 of them, relatively, and the function its own few."""
    one = torch.ones_like(z)
    if name == "none":
        return z, one, 0 * z, 0 * z
    if name == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype), 0 * z, 0 * z
    if name == "gelu":
        p, density = 0.5 * torch.special.erfc(-z / math.sqrt(2)), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        rel = (16 + 4 * (z * z).clamp(max=200)) * ULP
        return z * p, p + z * density, rel * (z * p).abs() + TINY * (1 + z.abs()), rel * (p + (z * density).abs()) + TINY * (1 + z.abs())
    c = math.sqrt(2 / math.pi)
    a, da = (z, one) if name == "silu" else (2 * c * (z + 0.044715 * z ** 3), 2 * c * (1 + 3 * 0.044715 * z * z))
    p, rest = torch.sigmoid(a), torch.sigmoid(-a)
    rel = (16 + 8 * a.abs().clamp(max=150)) * ULP
    return z * p, p + z * p * rest * da, rel * (z * p).abs() + TINY * (1 + z.abs()), rel * (p + (z * p * rest * da).abs()) + TINY * (1 + z.abs())


STEEPEST = 1.2                                                      # no derivative above is larger (1.13 and 1.10 are)


def product(x, w):
    """x w^T and what its sum of x.shape[1] terms in 32 bits may be off, each addition allowed twice a rounding."""
    return x @ w.t().contiguous(), 2 * (x.shape[1] + 2) * ULP * (x.abs() @ w.abs().t().contiguous())


def linear(x, w, bias, act, r):
    """z and y with what they may be off before they are rounded."""
    z, dz = product(x, w)
    if bias is not None:
        z = z + bias
        dz = dz + ULP * z.abs()
    a, _, da, _ = activation(z, act)
    y, dy = a, STEEPEST * dz + da
    if r is not None:
        y = y + r
        dy = dy + ULP * (y.abs() + dy)
    return z, dz, y, dy


def gated(x, wg, wu, act):
    (g, dg), (u, du) = product(x, wg), product(x, wu)
    a, _, da, _ = activation(g, act)
    da = da + STEEPEST * dg
    return g, dg, u, du, a * u, a.abs() * du + da * (u.abs() + du) + 2 * ULP * (a * u).abs()


def linear_grad(x, w, act, z, dy, type):
    """(dx, off), (dw, off), (dbias, off); the offs are before dx and dw are rounded, with dz rounded to the type where there is an activation."""
    _, slope, _, off = activation(z, act)
    dz = dy * slope
    off = dy.abs() * off + 2 * ULP * dz.abs()
    held = off + (stored(dz.abs() + off, type) if act != "none" else 0)
    dx, ox = product(dz, w.t().contiguous())
    dw, ow = product(dz.t().contiguous(), x.t().contiguous())
    ox, ow = 1.01 * ox + held @ w.abs(), 1.01 * ow + held.t().contiguous() @ x.abs()
    return (dx, ox), (dw, ow), (dz.sum(0), off.sum(0) + 2 * (len(dz) + 8) * ULP * (dz.abs() + off).sum(0))


def gated_grad(x, wg, wu, act, g, u, dy, type):
    """(dx, off), (dwg, off), (dwu, off) as above."""
    a, slope, oa, os = activation(g, act)
    out, dx, ox = [], 0, 0
    for d, off, w in ((dy * u * slope, (dy * u).abs() * os, wg), (dy * a, dy.abs() * oa, wu)):
        off = off + 3 * ULP * d.abs()
        held = off + stored(d.abs() + off, type)
        term, o = product(d, w.t().contiguous())
        dx, ox = dx + term, ox + 2.02 * o + held @ w.abs()          # (one sum of twice as many terms)
        dw, ow = product(d.t().contiguous(), x.t().contiguous())
        out.append((dw, 1.01 * ow + held.t().contiguous() @ x.abs()))
    return [(dx, ox)] + out


def block_norm(x, r, w_post, gate, group, scale, eps, w_pre):
    """r' and h in 64 bits with what they may be off before they are rounded; x and r may be None.  A row's squares: sixteen added one after another, then ten
    exchanges at most, 26 roundings of which rho has half; three of its own, and the products around it: 24."""
    if x is None:
        total, off = r, 0 * r
    else:
        u = x if w_post is None else x * torch.rsqrt((x * x).mean(1, keepdim=True) + eps) * w_post
        if gate is not None:
            u = u * gate[torch.arange(len(x), device=x.device) // group]
        total = scale * u + (0 if r is None else r)
        off = 24 * ULP * ((scale * u).abs() + (0 if r is None else r.abs()))
    if w_pre is None:
        return total, off, None, None
    rho = torch.rsqrt((total * total).mean(1, keepdim=True) + eps)
    h = total * rho * w_pre
    return total, off, h, rho * w_pre.abs() * off + h.abs() * (24 * ULP + off.norm(dim=1, keepdim=True) / total.norm(dim=1, keepdim=True).clamp(min=1e-300))


def block_norm_grad(x, r, w_post, gate, group, scale, eps, w_pre, dh, dr_out):
    """name -> (gradient, what it may be off before it is rounded): dr, dx, dw_pre, dw_post, dgate.  96 roundings of every term (of n 17, rho's with it, of the
    mean along a row 26 and rho's 17 again, of the factor rho 16, and the products) and, for a sum over rows, one a row."""
    rows, k = (dh if dh is not None else dr_out).shape
    device = (dh if dh is not None else dr_out).device
    few, many = 96 * ULP, 2 * (rows + 48) * ULP
    out = {}
    dr = torch.zeros((rows, k), dtype=torch.float64, device=device) if dr_out is None else dr_out
    terms = dr.abs()
    if dh is not None:
        rho = torch.rsqrt((r * r).mean(1, keepdim=True) + eps)
        dn, n = dh * w_pre, r * rho
        dr = dr + rho * (dn - n * (dn * n).mean(1, keepdim=True))
        terms = terms + rho * (dn.abs() + n.abs() * (dn * n).abs().mean(1, keepdim=True))
        out["dw_pre"] = ((dh * n).sum(0), many * (dh * n).abs().sum(0))
    out["dr"] = (dr, few * terms)
    if x is None:
        return out
    index = torch.arange(rows, device=device) // (group or rows)
    g = scale * (gate[index] if gate is not None else torch.ones_like(x))
    d, off = g * dr, g.abs() * few * terms
    if w_post is not None:
        rho = torch.rsqrt((x * x).mean(1, keepdim=True) + eps)
        m, d, off = x * rho, d * w_post, off * w_post.abs()
        out["dx"] = (rho * (d - m * (d * m).mean(1, keepdim=True)),
                     rho * (off + m.abs() * (off * m.abs()).mean(1, keepdim=True) + few * (d.abs() + m.abs() * (d * m).abs().mean(1, keepdim=True))))
        out["dw_post"] = ((g * dr * m).sum(0), ((g * m).abs() * (few * terms + many * dr.abs())).sum(0))
        u = m * w_post
    else:
        out["dx"], u = (d, off + few * d.abs()), x
    if gate is not None:
        part = torch.zeros_like(gate)
        out["dgate"] = (part.index_add(0, index, scale * dr * u), part.index_add(0, index, abs(scale) * u.abs() * (few * terms + many * dr.abs())))
    return out


def within(got, want, off, type):
    """Whether a result of the type is as near to `want` as its rounding and `off` allow; no NaN passes.  Numbers of 65520 and more, the middle between the largest
    FP16 number and the next, 2^16, that there would be, become infinite there."""
    got = got.double()
    near = (got - want).abs() <= rounded(want, off, type)
    if type == "f16":
        near |= torch.isinf(got) & (torch.sign(got) == torch.sign(want)) & (want.abs() + off >= 65520)
    return bool(torch.all(near))
