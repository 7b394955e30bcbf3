"""What a layer has between its projections and the operators of operators.py, as cases to be measured: the norms and the
position rotation of queries and keys ahead of attention, the experts' products and the gated activation between them, and
their gradients.

A case is a dict of plain values:
  kind    product | weight_gradient | gate | gate_gradient | rotate | rotate_gradient
  the first four  N tokens of K experts each out of E, the last `padded` of them without experts: rows [N * K] sorted by expert,
                  those of the padding behind all others, left as they are
  product, weight_gradient   width (of the rows that are multiplied), out_width, layout ("nk": a weight for each expert of
                  [out_width x width], as linear layers keep them; "kn": [width x out_width], which is also the gradient of
                  the rows of the other one)
  gate, gate_gradient        width (of the result; what goes in has gates and values side by side)
  rotate, rotate_gradient    tokens, padded (of which the last so many have no position), seqs, past (most tokens ahead of a
                  sequence's first one), mix (the lengths' own seed), heads, kv_heads, dim, rot (how much of a head is
                  rotated), interleaved (pairs are neighbours, not halves), norm, packed (q and k are columns of one
                  projection's output), pos_bits

Rows are bf16 normals, weights normals over the root of what they sum, norms' weights around 1. Experts are chosen as a router
does it, the K largest of E logits with a bias for each expert that makes some of them busier than others.

`own` chooses between the package's entry points and plain torch operations in 32 bits.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # one token's experts in a small model: launch and latency, a few weights from memory
        dict(name="product_token", kind="product", N=1, padded=0, E=16, K=4, width=2048, out_width=1024, layout="nk"),
        # a decode iteration on one of eight GPUs: every expert's weights for a few rows each
        dict(name="product_decode", kind="product", N=48, padded=0, E=8, K=2, width=4096, out_width=3584, layout="nk"),
        # a small prefill iteration over many small experts, the batch padded: some tens of rows to an expert
        dict(name="product_ragged", kind="product", N=541, padded=20, E=64, K=6, width=2048, out_width=2816, layout="nk"),
        # a prefill iteration of 8K tokens: a thousand rows to an expert
        dict(name="product_prefill", kind="product", N=8192, padded=0, E=64, K=8, width=4096, out_width=2048, layout="nk"),
        # the gradient of an expert's input in a training step: few large experts, a batch that is no round number
        dict(name="product_gradient", kind="product", N=2531, padded=19, E=8, K=2, width=7168, out_width=5120, layout="kn"),
        # the gradient of the weights: a small batch over small experts, and a training step's over large ones
        dict(name="weight_gradient_small", kind="weight_gradient", N=300, padded=7, E=16, K=4, width=2048, out_width=1024, layout="nk"),
        dict(name="weight_gradient", kind="weight_gradient", N=8192, padded=0, E=8, K=2, width=4096, out_width=7168, layout="nk"),
        # the activation of a decode iteration, and its gradient in a training step
        dict(name="gate_decode", kind="gate", N=64, padded=0, E=64, K=6, width=1408),
        dict(name="gate_gradient", kind="gate_gradient", N=8101, padded=91, E=64, K=8, width=1024),
        # queries and keys of a decode iteration, of a padded prefill iteration, and their gradient in a training step
        dict(name="rotate_decode", kind="rotate", tokens=48, padded=0, seqs=48, past=6000, mix=1, heads=64, kv_heads=8, dim=128,
             rot=128, interleaved=False, norm=True, packed=True, pos_bits=64),
        dict(name="rotate_prefill", kind="rotate", tokens=8101, padded=91, seqs=23, past=0, mix=2, heads=28, kv_heads=4, dim=128,
             rot=128, interleaved=False, norm=True, packed=True, pos_bits=64),
        dict(name="rotate_gradient", kind="rotate_gradient", tokens=16384, padded=0, seqs=4, past=0, mix=3, heads=32, kv_heads=8,
             dim=128, rot=128, interleaved=False, norm=True, packed=True, pos_bits=32),
    ]


MOST_FLOPS = 1.09e12     # the largest listed product
MOST_WEIGHTS = 1 << 30   # elements of all experts' weights
MOST_BYTES = 9e8         # of the rows that gates and rotations read and write


def draw(rng):
    def spread(lo, hi, multiple=1):
        v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
        return max(multiple, int(v / multiple + 0.5) * multiple)

    kind = rng.choice(("product", "product", "product", "product", "weight_gradient", "weight_gradient", "gate", "gate_gradient",
                       "rotate", "rotate", "rotate_gradient"))
    if kind.startswith("rotate"):
        heads, kv_heads, dim = rng.choice(((8, 2, 64), (16, 16, 64), (12, 4, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128),
                                           (8, 1, 128), (20, 20, 96), (24, 8, 80), (16, 2, 72)))
        tokens = spread(1, 16384)
        case = dict(kind=kind, tokens=tokens, padded=rng.choice((0, 0, tokens // 9)), seqs=min(tokens, spread(1, 64)),
                    past=rng.choice((0, spread(16, 30000))), mix=rng.randrange(1 << 30), heads=heads, kv_heads=kv_heads, dim=dim,
                    rot=rng.choice((dim, dim, dim, dim // 16 * 8)), interleaved=rng.random() < 0.3, norm=rng.random() < 0.8,
                    packed=rng.random() < 0.7, pos_bits=rng.choice((32, 64)))
        while work(case)["bytes"] > MOST_BYTES:
            case["tokens"] = case["tokens"] * 2 // 3
        case["seqs"], case["padded"] = min(case["tokens"], case["seqs"]), min(case["padded"], case["tokens"] // 9)
        return case
    N = spread(1, 16384)
    case = dict(kind=kind, N=N, padded=rng.choice((0, 0, N // 9)), E=rng.choice((8, 16, 64, 128, 160)))
    case["K"] = min(case["E"], rng.choice((1, 2, 2, 4, 6, 8, 8)))
    case["width"] = rng.choice((1024, 2048, 4096, 5120, 7168, spread(256, 8192, 8)))
    if kind.startswith("gate"):
        while work(case)["bytes"] > MOST_BYTES:
            case["N"] = case["N"] * 2 // 3
    else:
        case["out_width"] = rng.choice((1024, 1536, 2816, 3584, 4096, spread(256, 8192, 8)))
        case["layout"] = rng.choice(("nk", "nk", "kn"))
        while case["E"] * case["width"] * case["out_width"] > MOST_WEIGHTS:
            wider = "width" if case["width"] > case["out_width"] else "out_width"
            case[wider] = case[wider] // 16 * 8
        while work(case)["flops"] > MOST_FLOPS:
            case["N"] = case["N"] * 2 // 3
    case["padded"] = min(case["padded"], case["N"] // 9)
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(std=std, generator=g)


def _zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype, device=DEV)


def _expert_offsets(case, g):
    """The first row of each expert, and the number of all that have one."""
    N, E, K = case["N"], case["E"], case["K"]
    logits = torch.empty(N, E, device=DEV).normal_(generator=g) + 0.5 * torch.empty(E, device=DEV).normal_(generator=g)
    ids = torch.topk(logits, K, dim=1).indices[:N - case["padded"]]
    counts = torch.bincount(ids.flatten(), minlength=E)
    return torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)


def _expert_inputs(case, seed):
    g = _generator(seed)
    offsets = _expert_offsets(case, g)
    rows, W, kind = case["N"] * case["K"], case["width"], case["kind"]
    if kind == "gate":
        return dict(x=_normal(g, rows, 2 * W), limit=offsets[-1:], out=_zeros(rows, W))
    if kind == "gate_gradient":
        return dict(dout=_normal(g, rows, W), x=_normal(g, rows, 2 * W), limit=offsets[-1:], dx=_zeros(rows, 2 * W))
    O, kn = case["out_width"], case["layout"] == "kn"
    shape = (case["E"],) + ((W, O) if kn else (O, W))
    if kind == "product":
        return dict(A=_normal(g, rows, W), B=_normal(g, *shape, std=W ** -0.5), offsets=offsets, b_layout=int(kn), C=_zeros(rows, O))
    return dict(A=_normal(g, rows, W), dC=_normal(g, rows, O), offsets=offsets, b_layout=int(kn), dB=_zeros(*shape))


def _positions(case):
    """Of each token: sequences one behind the other, and padding."""
    rng = random.Random(case["mix"])
    parts = [rng.lognormvariate(0.0, 0.9) for _ in range(case["seqs"])]
    over = case["tokens"] - case["padded"] - case["seqs"]
    rows = [1 + max(0, int(over * p / sum(parts))) for p in parts]
    at = []
    for r in rows:
        past = rng.randrange(case["past"] + 1)
        at.extend(range(past, past + r))
    at = at[:case["tokens"] - case["padded"]]
    at.extend(range(case["tokens"] - case["padded"] - len(at)))
    return at + [-1] * case["padded"]


ROTATION_BASE = 10000.0
EPS = 1e-6


def _rotation(positions, rot):
    """A row for each position: the cosines of its angles, then their sines. In 64 bits up to the end, as far angles need."""
    angles = torch.arange(positions, dtype=torch.float64)[:, None] * ROTATION_BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([angles.cos(), angles.sin()], dim=1).float().to(DEV)


def _heads(case, g, rows):
    Hq, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    if case["packed"]:
        qkv = _normal(g, rows, Hq + 2 * Hk, D)
        return qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    return _normal(g, rows, Hq, D), _normal(g, rows, Hk, D)


def _rotate_inputs(case, seed):
    g = _generator(seed)
    T, Hq, Hk, D = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    at = _positions(case)
    q, k = _heads(case, g, T)
    weights = [(1 + _normal(g, D, std=0.1).float()).bfloat16() if case["norm"] else None for _ in range(2)]
    args = dict(q=q, k=k, positions=torch.tensor(at, dtype=torch.int64 if case["pos_bits"] == 64 else torch.int32, device=DEV),
                rotation=_rotation(max(at) + 1, case["rot"]), q_weight=weights[0], k_weight=weights[1], eps=EPS,
                interleaved=case["interleaved"])
    if case["kind"] == "rotate":
        return dict(args, q_out=_zeros(T, Hq, D), k_out=_zeros(T, Hk, D))
    args.update(dq=_normal(g, T, Hq, D), dk=_normal(g, T, Hk, D), dq_out=_zeros(T, Hq, D), dk_out=_zeros(T, Hk, D))
    if not case["norm"]:
        args.update(q=None, k=None)
    return args


def prepare(case, seed):
    args = _rotate_inputs(case, seed) if case["kind"].startswith("rotate") else _expert_inputs(case, seed)
    state = dict(kind=case["kind"], args=args)
    if "offsets" in args:
        state["at"] = args["offsets"].tolist()      # for the plain form, one product after the other
    return state


# ---- one pass -------------------------------------------------------------------------------------------------

def run(state):
    kind, args = state["kind"], state["args"]
    if own:
        import paper_2505_11329_amd as tw
        name = {"product": "expert_gemm", "weight_gradient": "expert_gemm_backward", "gate": "gated_silu",
                "gate_gradient": "gated_silu_backward", "rotate": "qk_norm_rope", "rotate_gradient": "qk_norm_rope_backward"}[kind]
        out = getattr(tw, name)(**args)
        return tuple(t for t in out if t is not None) if isinstance(out, tuple) else out
    if kind == "product":
        return _product(state["at"], **args)
    if kind == "weight_gradient":
        return _weight_gradient(state["at"], **args)
    return {"gate": _gate, "gate_gradient": _gate_gradient, "rotate": _rotate, "rotate_gradient": _rotate_gradient}[kind](**args)


def _product(at, A, B, offsets, b_layout, C):
    C = torch.zeros_like(C)
    for e in range(len(at) - 1):
        if at[e] < at[e + 1]:
            w = B[e].float()
            C[at[e]:at[e + 1]] = (A[at[e]:at[e + 1]].float() @ (w if b_layout else w.t())).to(C.dtype)
    return C


def _weight_gradient(at, A, dC, offsets, b_layout, dB):
    dB = torch.zeros_like(dB)
    for e in range(len(at) - 1):
        if at[e] < at[e + 1]:
            x, d = A[at[e]:at[e + 1]].float(), dC[at[e]:at[e + 1]].float()
            dB[e] = ((x.t() @ d) if b_layout else (d.t() @ x)).to(dB.dtype)
    return dB


def _live(like, limit):
    return torch.arange(like.shape[0], device=like.device)[:, None] < limit


def _gate(x, limit, out):
    g, u = x.float().chunk(2, dim=1)
    return torch.where(_live(x, limit), g / (1 + torch.exp(-g)) * u, 0.0).to(out.dtype)


def _gate_gradient(dout, x, limit, dx):
    g, u = x.float().chunk(2, dim=1)
    d = dout.float()
    s = 1 / (1 + torch.exp(-g))
    both = torch.cat([d * u * s * (1 + g * (1 - s)), d * g * s], dim=1)
    return torch.where(_live(x, limit), both, 0.0).to(dx.dtype)


def _turned(x, positions, rotation, interleaved, back):
    """x [T, H, D] with its first columns rotated by the tokens' angles, or back."""
    cos, sin = rotation[positions.clamp(min=0).long()].to(x.dtype)[:, None].chunk(2, dim=2)
    if back:
        sin = -sin
    rot = 2 * cos.shape[2]
    if interleaved:
        first, second = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        first, second = x[..., :rot // 2], x[..., rot // 2:rot]
    first, second = first * cos - second * sin, second * cos + first * sin
    turned = torch.stack([first, second], dim=3).flatten(2) if interleaved else torch.cat([first, second], dim=2)
    return torch.cat([turned, x[..., rot:]], dim=2)


def _rotate_one(x, weight, positions, rotation, eps, interleaved, out):
    z = x.float()
    if weight is not None:
        z = z * torch.rsqrt(z.square().mean(2, keepdim=True) + eps) * weight.float()
    y = _turned(z, positions, rotation, interleaved, False)
    return torch.where((positions >= 0)[:, None, None], y, 0.0).to(out.dtype)


def _rotate(q, k, positions, rotation, q_weight, k_weight, eps, interleaved, q_out, k_out):
    return (_rotate_one(q, q_weight, positions, rotation, eps, interleaved, q_out),
            _rotate_one(k, k_weight, positions, rotation, eps, interleaved, k_out))


def _rotate_gradient_one(dy, x, weight, positions, rotation, eps, interleaved, out):
    has = (positions >= 0)[:, None, None]
    dz = _turned(dy.float(), positions, rotation, interleaved, True)
    if weight is None:
        return torch.where(has, dz, 0.0).to(out.dtype), None
    xf = x.float()
    r = torch.rsqrt(xf.square().mean(2, keepdim=True) + eps)
    n = xf * r
    dweight = torch.where(has, dz * n, 0.0).sum((0, 1), dtype=torch.float64).float()
    g = dz * weight.float()
    return torch.where(has, r * (g - n * (g * n).mean(2, keepdim=True)), 0.0).to(out.dtype), dweight


def _rotate_gradient(dq, dk, q, k, positions, rotation, q_weight, k_weight, eps, interleaved, dq_out, dk_out):
    dx_q, dw_q = _rotate_gradient_one(dq, q, q_weight, positions, rotation, eps, interleaved, dq_out)
    dx_k, dw_k = _rotate_gradient_one(dk, k, k_weight, positions, rotation, eps, interleaved, dk_out)
    return tuple(t for t in (dx_q, dx_k, dw_q, dw_k) if t is not None)


# ---- what a pass cannot do without, and its results in 64 bits --------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind.startswith("rotate"):
        T, H = case["tokens"] - case["padded"], case["heads"] + case["kv_heads"]
        moved = 2 if kind == "rotate" or not case["norm"] else 3
        return dict(bytes=2 * moved * T * H * case["dim"] + T * (4 * case["rot"] + case["pos_bits"] // 8),
                    flops=(6 if kind == "rotate" else 14) * T * H * case["dim"])
    rows, W, E = (case["N"] - case["padded"]) * case["K"], case["width"], case["E"]
    if kind.startswith("gate"):
        return dict(bytes=2 * rows * W * (3 if kind == "gate" else 5), flops=(5 if kind == "gate" else 10) * rows * W)
    O = case["out_width"]
    # of few rows, the experts that have one: as many as choices at random meet
    met = E if kind == "weight_gradient" else max(min(E, case["K"]), round(E * (1 - (1 - case["K"] / E) ** (case["N"] - case["padded"]))))
    return dict(bytes=2 * (rows * (W + O) + met * W * O), flops=2 * rows * W * O)


def exact(case, seed):
    state = prepare(case, seed)
    kind, args = case["kind"], state["args"]
    if kind in ("product", "weight_gradient"):
        at, kn = state["at"], args["b_layout"]
        out = torch.zeros((args["C"] if kind == "product" else args["dB"]).shape, dtype=torch.float64, device=DEV)
        for e, (lo, hi) in enumerate(zip(at, at[1:])):
            x = args["A"][lo:hi].double()
            if kind == "product":
                w = args["B"][e].double()
                out[lo:hi] = torch.mm(x, w if kn else w.t().contiguous())
            else:
                d = args["dC"][lo:hi].double()
                out[e] = torch.mm(x.t().contiguous(), d) if kn else torch.mm(d.t().contiguous(), x)
        return out
    if kind.startswith("gate"):
        W, live = case["width"], int(args["limit"])
        x = args["x"][:live].double()
        g, u = x[:, :W], x[:, W:]
        s = torch.sigmoid(g)
        if kind == "gate":
            out = torch.zeros(args["out"].shape, dtype=torch.float64, device=DEV)
            out[:live] = g * s * u
            return out
        out = torch.zeros(args["dx"].shape, dtype=torch.float64, device=DEV)
        d = args["dout"][:live].double()
        out[:live, :W] = d * u * (s + g * s * (1 - s))
        out[:live, W:] = d * g * s
        return out
    return _exact_rotate(case, args)


def _exact_rotate(case, args):
    """The rotation as complex numbers; a head's gradient through its norm from the definition."""
    T, rot = case["tokens"] - case["padded"], case["rot"]
    table = args["rotation"].double()[args["positions"][:T].long()]
    turn = torch.complex(table[:, :rot // 2], table[:, rot // 2:])[:, None]

    def turned(x, by):
        x = x.clone()
        if case["interleaved"]:
            z = torch.view_as_complex(x[..., :rot].reshape(x.shape[:2] + (rot // 2, 2)).contiguous()) * by
            x[..., :rot] = torch.view_as_real(z).flatten(2)
        else:
            z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * by
            x[..., :rot // 2], x[..., rot // 2:rot] = z.real, z.imag
        return x

    grads, results, weights = case["kind"] == "rotate_gradient", [], []
    for name in ("q", "k"):
        heads, D = case["heads" if name == "q" else "kv_heads"], case["dim"]
        result = torch.zeros(case["tokens"], heads, D, dtype=torch.float64, device=DEV)
        dweight = torch.zeros(D, dtype=torch.float64, device=DEV)
        w = args[name + "_weight"].double() if case["norm"] else None
        for lo in range(0, T, 2048):        # some rows at a time
            rows = slice(lo, min(lo + 2048, T))
            x = args[name][rows].double() if args[name] is not None else None
            if w is not None:
                size = (x.square().sum(2, keepdim=True) / D + EPS).sqrt()
            if not grads:
                result[rows] = turned(x / size * w if w is not None else x, turn[rows])
                continue
            d = turned(args["d" + name][rows].double(), turn[rows].conj())
            if w is not None:
                dweight += (d * x / size).sum((0, 1))
                along = (d * w * x).sum(2, keepdim=True)
                d = d * w / size - x * along / (D * size ** 3)
            result[rows] = d
        results.append(result)
        weights.append(dweight)
    return tuple(results + (weights if grads and case["norm"] else []))
