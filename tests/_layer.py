"""Plain implementations, in 64 bits, of a layer's norm, rotation and attention over prompts, with what the roundings of fp32 and of 16-bit results may make."""
import fractions
import math

import torch

from _serving import half_step

NEG = float("-inf")
F32_STEP = 2.0 ** -24
PI = fractions.Fraction("3.14159265358979323846264338327950288419716939937510582097")


def least(dtype):
    """Half of the distance of the type's smallest numbers."""
    f = torch.finfo(dtype)
    return f.tiny * f.eps / 2


def norm_reference(x, weight, eps, residual):
    """h and y, float64."""
    h = x.double() if residual is None else x.double() + residual.double()
    return h, h / torch.sqrt(h.square().mean(-1, keepdim=True) + eps) * weight.double()


def norm_tolerance(y, dtype):
    """h, the factor, its product with h and that with the weight: a rounding each, and one more for the factor, which is that of h as it was rounded."""
    return y.abs() * (half_step(dtype) * (1 + 2.0 ** -8) + 5 * F32_STEP) + least(dtype)


def blocks_of(y, n):
    """y cut into blocks of n along its last dimension, and for each element the largest size of its block."""
    parts = y.split(n, -1)
    top = torch.stack([p.abs().max(-1).values for p in parts], -1)
    return top, torch.cat([t.unsqueeze(-1).expand(p.shape) for t, p in zip(top.unbind(-1), parts)], -1)


def turned_reference(x, positions, dim, frequencies, neighbours, magnitude):
    """x [tokens][heads][D] float64, turned, and the tolerance of an output of its type: angles as fractions of a turn without any rounding."""
    y = x.double().clone()
    tol = torch.zeros_like(y)
    turns = [[float((int(p) * fractions.Fraction(float(f)) / (2 * PI)) % 1) for f in frequencies] for p in positions]
    angle = 2 * math.pi * torch.tensor(turns, dtype=torch.float64, device=x.device).reshape(len(positions), 1, dim // 2)
    first = torch.arange(0, dim, 2, device=x.device) if neighbours else torch.arange(dim // 2, device=x.device)
    second = first + (1 if neighbours else dim // 2)
    a, b = x[..., first].double(), x[..., second].double()
    y[..., first] = magnitude * (a * torch.cos(angle) - b * torch.sin(angle))
    y[..., second] = magnitude * (a * torch.sin(angle) + b * torch.cos(angle))
    # Sine and cosine: the angle's argument |x| <= pi / 4 with two roundings, 9.4e-8; the series' rest, 2.5e-8; its last additions, 2^-23; the fractions of a turn, 1e-9; in all below
    # 2^-21.  Their products with the magnitude and with the elements, and the sum: a rounding each.
    size = (a.abs() + b.abs()) * abs(magnitude) * (2.0 ** -21 + 4 * F32_STEP)
    for at in (first, second):
        tol[..., at] = size + y[..., at].abs() * half_step(x.dtype) * (1 + 2.0 ** -8) + least(x.dtype)
    return y, tol


def prompt_reference(q, k, v, starts, scale):
    """out, lse, and how far 16-bit weights and fp32 sums may be off in each, float64; rows of no sequence hold NaN."""
    rows, H, D = q.shape
    G = H // k.shape[1]
    out = torch.full((rows, H, D), float("nan"), dtype=torch.float64, device=q.device)
    lse = torch.full((rows, H), float("nan"), dtype=torch.float64, device=q.device)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    u = half_step(q.dtype)
    for a, z in zip(starts, starts[1:]):
        if not 0 <= a < z <= rows:
            continue
        n = z - a
        seen = torch.ones((n, n), dtype=torch.bool, device=q.device).tril()
        for h in range(H):
            K, V = k[a:z, h // G].double(), v[a:z, h // G].double()
            x = torch.where(seen, (q[a:z, h].double() @ K.T.contiguous()) * scale, NEG)
            size = torch.where(seen, q[a:z, h].double().abs() @ K.abs().T.contiguous() * scale, 0.0).max(1).values
            top = x.max(1).values
            p = torch.where(seen, torch.exp(x - top[:, None]), 0.0)
            total = p.sum(1)
            odd = ~torch.isfinite(V)
            clean = torch.where(odd, 0.0, V)
            o, mean = p @ clean / total[:, None], p @ clean.abs() / total[:, None]
            if bool(odd.any()):                             # only for the rows that see them
                for j in torch.nonzero(odd.any(1))[:, 0].tolist():
                    o[j:] += torch.where(odd[j], p[j:, j:j + 1] * V[j], 0.0) / total[j:, None]
            out[a:z, h], lse[a:z, h] = o, top + torch.log(total)
            # scores: sums of D products in fp32, the scale's rounding, the exponent's argument and the exponential; weights and their sum as rounded: a mean of
            # other weights, off by u of |v - out|; sums of n terms and their rescalings in fp32; of halves, weights below 2^-27 of the largest lose 2^-38 of it
            d = (D + 4) * F32_STEP * size + 4 * 2.0 ** -23 * (1 + size)
            s = (n + 64) * 2.0 ** -23
            lost = n * 2.0 ** -37 * clean.abs().max() if q.dtype == torch.float16 else 0.0
            own = torch.nan_to_num(o, 0, 0, 0).abs()
            tol[a:z, h] = u * (1 + 2.0 ** -8) * own + (mean + own) * (u * (1 + 4 * u) + 2 * d + s)[:, None] + lost + least(q.dtype)
            tol_lse[a:z, h] = d + s + lse[a:z, h].abs() * 2.0 ** -22
    return out, lse, tol, tol_lse
