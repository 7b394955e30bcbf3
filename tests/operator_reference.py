"""Plain 64-bit forms of attention and of the experts' operators, and how far the kernels may be from them. A result in
bf16 is off by half a step, 2^-8 of its value; what else the kernels round is counted beside each bound."""
import math

import torch

BF16 = 2.0 ** -8        # half a step, relative
F32 = 2.0 ** -24


def offsets(lengths, start=0):
    at = [start]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32)


def attention(q, k, v, q_offsets, k_offsets, causal, scale):
    """(out, lse, out's bound, lse's bound), float64 on q's device; rows of no sequence are NaN.

    Bounds, with A = sum_j w_j |v_j|, w the softmax: the score of a key is a sum of D products in fp32, in any order: off by
    at most D F32 sum |q k| scale, plus two roundings of the scaled score and one of the maximum (4 F32 |s| in all); such
    an error e changes a weight by a factor of 1 +- e and the total by as much, 2 e in all. 2^x and the division add
    at most 2^-21. The product with v rounds each p to bf16 (BF16 A), sums in fp32 (keys F32 A), and the result is rounded to
    bf16. lse: the score's error, and log2, the sum and the scaling by ln 2 in fp32 (keys + 8 roundings)."""
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    nan = dict(dtype=torch.float64, device=q.device)
    out, tol = torch.full((T, Hq, D), math.nan, **nan), torch.full((T, Hq, D), math.nan, **nan)
    lse, tol_lse = torch.full((T, Hq), math.nan, **nan), torch.full((T, Hq), math.nan, **nan)
    qo, ko = q_offsets.tolist(), k_offsets.tolist()
    for b in range(len(qo) - 1):
        rows, keys = slice(qo[b], qo[b + 1]), slice(ko[b], ko[b + 1])
        lq, lk = qo[b + 1] - qo[b], ko[b + 1] - ko[b]
        if lq == 0:
            continue
        seen = torch.ones(lq, lk, dtype=torch.bool, device=q.device)
        if causal:
            seen = seen.tril(lk - lq)
        for h in range(Hq):
            x, y, z = (t.double() for t in (q[rows, h], k[keys, h // G], v[keys, h // G]))
            s = torch.where(seen, (x @ y.T) * scale, -math.inf)
            size = torch.where(seen, (x.abs() @ y.abs().T) * scale, 0.0)
            m = s.amax(1, keepdim=True) if lk else torch.full((lq, 1), -math.inf, **nan)
            p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
            total = p.sum(1, keepdim=True)
            some = seen.any(1, keepdim=True)
            w = torch.where(some, p / total, 0.0)
            w = torch.where(seen, w, 0.0)
            # a weight of 0 where a key is hidden must not meet its value
            o = torch.zeros(lq, D, **nan)
            A = torch.zeros(lq, D, **nan)
            if lk:
                clean = torch.nan_to_num(z, 0.0, 0.0, 0.0)
                o, A = w @ clean, w @ clean.abs()
                for j in torch.nonzero(~torch.isfinite(z).all(1)).flatten().tolist():
                    o += torch.where(seen[:, j:j + 1] & ~torch.isfinite(z[j]), z[j], 0.0)
            e = (D * F32 * size.amax(1, keepdim=True) if lk else 0.0) + 4 * F32 * torch.nan_to_num(m.abs(), 0.0, 0.0, 0.0)
            out[rows, h] = o
            tol[rows, h] = BF16 * o.abs() + (BF16 + 2 * e + 2.0 ** -21 + lk * F32) * A * (1 + BF16)
            lse[rows, h] = (m + total.log()).squeeze(1)
            tol_lse[rows, h] = (e + F32 * (lk + 8) * (1 + m.abs().nan_to_num(0.0, 0.0, 0.0))).squeeze(1)
    return out, lse, tol, tol_lse


def assert_close(got, want, tol, what):
    got = got.double()
    assert got.shape == want.shape, what
    same = (got == want) | (torch.isnan(got) & torch.isnan(want)) | ((got - want).abs() <= tol)
    if not bool(same.all()):
        at = tuple(torch.nonzero(~same)[0].tolist())
        raise AssertionError("%s: %d of %d off; first at %s: %r, expected %r within %r"
                             % (what, int((~same).sum()), same.numel(), at, float(got[at]), float(want[at]), float(tol[at])))


def sort(ids, E):
    """(order, position, offsets) as lists."""
    flat = ids.flatten().tolist()
    buckets = [[] for _ in range(E + 1)]
    for pair, e in enumerate(flat):
        buckets[e if 0 <= e < E else E].append(pair)
    order = [pair for b in buckets for pair in b]
    offs = [0]
    for b in buckets[:E]:
        offs.append(offs[-1] + len(b))
    position = [-1] * len(flat)
    for s, pair in enumerate(order[:offs[E]]):
        position[pair] = s
    return order, position, offs


def combine(y, position, weights):
    """(out, bound): K products summed in fp32, then rounded to bf16."""
    N, K = position.shape
    out = torch.zeros(N, y.shape[1], dtype=torch.float64, device=y.device)
    size = torch.zeros_like(out)
    for k in range(K):
        has = (position[:, k] >= 0) & (position[:, k] < y.shape[0])
        rows = y[position[has, k].long()].double()
        if weights is not None:
            rows = rows * weights[has, k, None].double()
        out[has] += rows
        size[has] += rows.abs()
    return out, BF16 * out.abs() + (K + 1) * F32 * size


def combine_backward(dout, y, position, weights):
    """(dy, dy's bound, dw, dw's bound): a product in fp32 rounded to bf16; H products summed in fp32. Rows of dy that no
    pair has are NaN."""
    N, K = position.shape
    H = y.shape[1]
    dy = torch.full(y.shape, math.nan, dtype=torch.float64, device=y.device)
    dw = torch.zeros(N, K, dtype=torch.float64, device=y.device)
    size = torch.zeros_like(dw)
    for k in range(K):
        has = (position[:, k] >= 0) & (position[:, k] < y.shape[0])
        at, d = position[has, k].long(), dout[has].double()
        dy[at] = weights[has, k, None].double() * d
        dw[has, k] = (y[at].double() * d).sum(1)
        size[has, k] = (y[at].double() * d).abs().sum(1)
    return dy, (BF16 + 2 * F32) * dy.abs(), dw, (H + 2) * F32 * size
