"""Plain 64-bit forms of the experts' products, the gated activation and the norms and rotation of queries and keys, their
gradients, and how far the kernels may be from them. Half a step of a type, relative: bf16 2^-8, fp32 2^-24."""
import math

import torch

BF16 = 2.0 ** -8
F32 = 2.0 ** -24
TINY = 2.0 ** -126      # smaller results may be 0


def rows_of(offsets, rows):
    """(expert, first row, last row + 1) as the offsets are read: inside the tensor, and ascending."""
    at, found = 0, []
    for e, o in enumerate(offsets.tolist()):
        upto = max(at, min(max(o, 0), rows))
        if e:
            found.append((e - 1, at, upto))
        at = upto
    return found


# Products of bf16 are exact in fp32. Their K sums in fp32 are off by at most a step of what is summed each, whatever the order and
# whether the adders round or cut off (2 F32); then bf16.
def product(A, B, offsets, kn):
    """(out, bound); rows without an expert are NaN."""
    rows, K = A.shape
    N = B.shape[2 if kn else 1]
    out = torch.full((rows, N), math.nan, dtype=torch.float64, device=A.device)
    tol = torch.full_like(out, math.nan)
    for e, lo, hi in rows_of(offsets, rows):
        if lo < hi:
            w = B[e].double() if kn else B[e].double().t().contiguous()
            x = A[lo:hi].double()
            out[lo:hi] = x @ w
            tol[lo:hi] = BF16 * out[lo:hi].abs() + 2 * (K + 1) * F32 * (x.abs() @ w.abs())
    return out, tol


def weight_gradient(A, dC, offsets, E, kn):
    rows, K = A.shape
    N = dC.shape[1]
    out = torch.zeros((E, K, N) if kn else (E, N, K), dtype=torch.float64, device=A.device)
    tol = torch.zeros_like(out)
    for e, lo, hi in rows_of(offsets, rows):
        if lo < hi:
            x, d = A[lo:hi].double(), dC[lo:hi].double()
            if not kn:
                x, d = d, x
            out[e] = x.t().contiguous() @ d
            tol[e] = BF16 * out[e].abs() + 2 * (hi - lo + 1) * F32 * (x.abs().t().contiguous() @ d.abs())
    return out, tol


# s = 1 / (1 + exp(-g)): the exponent's argument is off by F32 |g|, exp2 and the reciprocal by a step (2 F32) each, the sum by F32:
# s by (|g| + 8) F32 of it. Two products more, and bf16. exp2 may give 0 below 2^-126.
def gate(x):
    F = x.shape[1] // 2
    g, u = x[:, :F].double(), x[:, F:].double()
    out = g * torch.sigmoid(g) * u
    return out, BF16 * out.abs() + (g.abs() + 10) * F32 * out.abs() * (1 + BF16) + TINY * (1 + (g * u).abs())


# The factor s (1 + g (1 - s)) is s + gs (1 - s): s and gs off by (|g| + 9) F32 of them, 1 - s by that and its own rounding.
def gate_backward(dout, x):
    F = x.shape[1] // 2
    g, u, d = x[:, :F].double(), x[:, F:].double(), dout.double()
    s = torch.sigmoid(g)
    dg, du = d * u * (s + g * s * (1 - s)), d * g * s
    size = (g.abs() + 10) * s + 2 * (g.abs() + 10) * g.abs() * s
    tol_g = BF16 * dg.abs() + (1 + BF16) * F32 * (d * u).abs() * size + 3 * F32 * dg.abs() + TINY * (1 + (d * u).abs() * (1 + g.abs()))
    tol_u = BF16 * du.abs() + (g.abs() + 12) * F32 * du.abs() * (1 + BF16) + TINY * (1 + (d * g).abs())
    return torch.cat([dg, du], 1), torch.cat([tol_g, tol_u], 1)


def table(positions, rot, base=10000.0):
    angles = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([angles.cos(), angles.sin()], 1).float()


def turned(x, cos, sin, interleaved, size=False):
    """x [T, H, D] with its pairs turned; with `size`, the sums of what is added, without their signs."""
    half = cos.shape[-1]
    y = x.clone()
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    if size:
        a, b, cos, sin = a.abs(), b.abs(), cos.abs(), sin.abs()
        y = y.abs()
        first, second = a * cos + b * sin, b * cos + a * sin
    else:
        first, second = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = first, second
    else:
        y[..., :half], y[..., half:2 * half] = first, second
    return y


def _angles(positions, rotation):
    has = (positions >= 0) & (positions < rotation.shape[0])
    t = rotation.double()[torch.where(has, positions, 0).long()]
    half = rotation.shape[1] // 2
    return has, t[:, None, :half], t[:, None, half:]


# The mean of D squares: D F32 and its own roundings; the root and the quotient a step each, halved or not: (D + 8) F32. Two products,
# then of a turned column two products and a sum.
def norm_rope(x, weight, positions, rotation, eps, interleaved):
    """(y, bound) [T, H, D]; padding is NaN."""
    D = x.shape[2]
    z = x.double()
    if weight is not None:
        z = z / torch.sqrt(z.square().mean(2, keepdim=True) + eps) * weight.double()
    y, size, has = z, z.abs(), torch.ones(x.shape[0], dtype=torch.bool, device=x.device)
    if rotation is not None:
        has, cos, sin = _angles(positions, rotation)
        y, size = turned(z, cos, sin, interleaved), turned(z, cos, sin, interleaved, size=True)
    tol = BF16 * y.abs() + (1 + BF16) * (D + 16) * F32 * size + TINY
    keep = has[:, None, None]
    return torch.where(keep, y, math.nan), torch.where(keep, tol, math.nan)


# dz as above without the norm: 4 F32 of its size. Both means: D F32 more; the difference by its own rounding. The weights' gradient:
# a sum of T x H such terms in fp32, in any order.
def norm_rope_backward(dy, x, weight, positions, rotation, eps, interleaved):
    """(dx, bound, dweight, bound); dx of padding is NaN."""
    T, H, D = dy.shape
    dz = dy.double()
    size, has = dz.abs(), torch.ones(T, dtype=torch.bool, device=dy.device)
    if rotation is not None:
        has, cos, sin = _angles(positions, rotation)
        dz, size = turned(dz, cos, -sin, interleaved), turned(dz, cos, sin, interleaved, size=True)
    keep = has[:, None, None]
    if weight is None:
        return torch.where(keep, dz, math.nan), torch.where(keep, BF16 * dz.abs() + 5 * F32 * size + TINY, math.nan), None, None
    xd, w = x.double(), weight.double()
    r = 1 / torch.sqrt(xd.square().mean(2, keepdim=True) + eps)
    g, g_size = dz * w, size * w.abs()
    dx = r * (g - xd * r * r * (g * xd).mean(2, keepdim=True))
    all_ = r * (g_size + xd.abs() * r * r * (g_size * xd.abs()).mean(2, keepdim=True))
    tol = BF16 * dx.abs() + (1 + BF16) * (4 * D + 48) * F32 * all_ + TINY
    terms, t_size = torch.where(keep, dz * xd * r, 0.0), torch.where(keep, size * xd.abs() * r, 0.0)
    return (torch.where(keep, dx, math.nan), torch.where(keep, tol, math.nan), terms.sum((0, 1)),
            (T * H + D + 24) * F32 * t_size.sum((0, 1)))
