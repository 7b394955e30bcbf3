"""Attention over packed sequences, and tokens sorted by expert and back, as cases to be measured: what a layer has
between its GEMMs and the fused step, from a batch of single decode tokens to the second split of a long prompt.

A case is a dict of plain values:
  kind    attention | sort | dispatch | combine | combine_backward
  attention   form (how the sequences' lengths are drawn, see lengths()), seqs, tokens (query rows of all sequences),
              past (most keys ahead of a sequence's first query row), mix (the lengths' own seed), heads, kv_heads, dim,
              causal, packed (q, k, v are columns of one projection's output), tail (query rows behind the last sequence)
  the others  N tokens, padded (of which the last so many have no expert), E experts, K experts a token, and
              H hidden size (all but sort), id_bits (sort), weighted (combine)

Inputs are bf16 normals, router weights a softmax over the chosen experts' logits in fp32. Experts are chosen as a
router does it, the K largest of E logits with a bias for each expert that makes some of them busier than others.

`own` chooses between the package's entry points and plain torch operations in 32 bits.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # one short prompt of a small model: launch and latency
        dict(name="attention_short", kind="attention", form="prompts", seqs=1, tokens=83, past=0, mix=1, heads=8, kv_heads=2,
             dim=64, causal=True, packed=True, tail=0),
        # one decode iteration: a token each of 48 requests, keys of up to 6K tokens
        dict(name="attention_decode", kind="attention", form="chunks", seqs=48, tokens=48, past=6000, mix=2, heads=64,
             kv_heads=8, dim=128, causal=True, packed=False, tail=0),
        # a prefill iteration over requests of different lengths, the batch padded to a whole number of rows
        dict(name="attention_packed", kind="attention", form="prompts", seqs=23, tokens=8101, past=0, mix=3, heads=32,
             kv_heads=8, dim=128, causal=True, packed=True, tail=91),
        # the last of a long prompt's splits: its rows attend to the keys of the splits before it
        dict(name="attention_suffix", kind="attention", form="chunks", seqs=1, tokens=4096, past=12288, mix=4, heads=64,
             kv_heads=8, dim=128, causal=True, packed=False, tail=0),
        # routing of one decode iteration
        dict(name="sort_decode", kind="sort", N=64, padded=0, E=64, K=6, id_bits=64),
        # routing of a prefill iteration of 16K tokens
        dict(name="sort_prefill", kind="sort", N=16384, padded=133, E=128, K=8, id_bits=32),
        # the rows of a decode iteration, and of a prefill iteration, on their way to the experts
        dict(name="dispatch_decode", kind="dispatch", N=48, padded=0, E=8, K=2, H=4096),
        dict(name="dispatch_prefill", kind="dispatch", N=8101, padded=91, E=64, K=6, H=4096),
        # the experts' results back, weighted; a wide model with few experts
        dict(name="combine_prefill", kind="combine", N=16384, padded=0, E=8, K=2, H=8192, weighted=True),
        # the gradient of the dispatch: the same sum without weights, a hidden size and a batch that are no round numbers
        dict(name="dispatch_gradient", kind="combine", N=2531, padded=19, E=128, K=8, H=5120, weighted=False),
        # the gradient of the weighted sum: a small batch, and a training step's
        dict(name="combine_gradient_small", kind="combine_backward", N=300, padded=7, E=16, K=4, H=2048),
        dict(name="combine_gradient", kind="combine_backward", N=8192, padded=0, E=64, K=8, H=4096),
    ]


MOST_FLOPS = 1.9e12      # the largest listed attention


def draw(rng):
    def spread(lo, hi, multiple=1):
        v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
        return max(multiple, int(v / multiple + 0.5) * multiple)

    kind = rng.choice(("attention", "attention", "attention", "sort", "dispatch", "combine", "combine_backward"))
    if kind == "attention":
        heads, kv_heads, dim = rng.choice(((8, 2, 64), (16, 16, 64), (12, 4, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128),
                                           (8, 1, 128), (20, 20, 96), (24, 8, 80), (16, 2, 72)))
        form, causal = rng.choice((("prompts", True), ("prompts", True), ("prompts", False), ("chunks", True),
                                   ("chunks", True), ("tokens", True), ("tokens", True)))
        seqs = spread(1, 64)
        case = dict(kind=kind, form="prompts" if form == "prompts" else "chunks", seqs=seqs,
                    tokens=seqs * rng.choice((1, 1, 2, 4)) if form == "tokens" else max(seqs, spread(1, 8192)),
                    past=0 if form == "prompts" else spread(16, 16384), mix=rng.randrange(1 << 30), heads=heads,
                    kv_heads=kv_heads, dim=dim, causal=causal, packed=form == "prompts" and rng.random() < 0.5,
                    tail=rng.choice((0, 0, 1, 37)))
        while work(case)["flops"] > MOST_FLOPS:
            case["tokens"] = max(seqs, case["tokens"] * 2 // 3)
            case["past"] = case["past"] * 2 // 3
        return case
    N = spread(1, 16384)
    case = dict(kind=kind, N=N, padded=rng.choice((0, 0, N // 9)), E=rng.choice((8, 16, 64, 128, 160, 256)))
    case["K"] = min(case["E"], rng.choice((1, 2, 2, 4, 6, 8, 8)))
    if kind == "sort":
        return dict(case, id_bits=rng.choice((32, 64)))
    case["H"] = rng.choice((2048, 4096, 5120, 7168, 8192, spread(512, 8192, 8)))
    while case["N"] * case["K"] * case["H"] > 8192 * 8 * 4096:
        case["N"] = case["N"] * 2 // 3
    case["padded"] = min(case["padded"], case["N"] // 9)
    return dict(case, weighted=rng.random() < 0.7) if kind == "combine" else case


def lengths(case):
    """Query rows and keys of each sequence. prompts: every key's row is a query; chunks: a sequence's query rows are
    the last of its keys, after up to `past` others (all of them where there is one sequence)."""
    rng = random.Random(case["mix"])
    parts = [rng.lognormvariate(0.0, 0.9) for _ in range(case["seqs"])]
    over = case["tokens"] - case["seqs"]
    rows = [1 + int(over * p / sum(parts)) for p in parts]
    rows[-1] += case["tokens"] - sum(rows)
    if case["form"] == "prompts":
        return rows, rows
    past = [case["past"]] if case["seqs"] == 1 else [rng.randrange(case["past"] + 1) for _ in rows]
    return rows, [r + p for r, p in zip(rows, past)]


# ---- inputs ---------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=g)


def _offsets(rows):
    at = [0]
    for r in rows:
        at.append(at[-1] + r)
    return torch.tensor(at, dtype=torch.int32, device=DEV)


def _attention_inputs(case, seed):
    g = _generator(seed)
    rows, keys = lengths(case)
    Hq, Hk, D, T, Tk = case["heads"], case["kv_heads"], case["dim"], sum(rows) + case["tail"], sum(keys)
    if case["packed"]:
        qkv = _normal(g, T, Hq + 2 * Hk, D)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    else:
        q, k, v = _normal(g, T, Hq, D), _normal(g, Tk, Hk, D), _normal(g, Tk, Hk, D)
    return dict(q=q, k=k, v=v, q_offsets=_offsets(rows), k_offsets=_offsets(keys), causal=case["causal"],
                out=torch.zeros(T, Hq, D, dtype=torch.bfloat16, device=DEV), lse=torch.zeros(T, Hq, device=DEV))


def _routing(case, seed):
    """The experts of each token and their weights, as a router gives them, and the generator."""
    g = _generator(seed)
    N, E, K = case["N"], case["E"], case["K"]
    logits = torch.empty(N, E, device=DEV).normal_(generator=g) + 0.5 * torch.empty(E, device=DEV).normal_(generator=g)
    top, ids = torch.topk(logits, K, dim=1)
    ids[N - case["padded"]:] = -1
    return ids, torch.softmax(top, dim=1), g


def _positions(ids, E):
    """The sorted place of each pair of a token and an expert, -1 where it has none."""
    flat = ids.flatten()
    valid = (flat >= 0) & (flat < E)
    order = torch.sort(torch.where(valid, flat, E), stable=True).indices
    position = torch.empty_like(order)
    position[order] = torch.arange(order.numel(), device=order.device)
    return torch.where(valid, position, -1).to(torch.int32).view(ids.shape)


def _expert_inputs(case, seed):
    ids, weights, g = _routing(case, seed)
    N, E, K, kind = case["N"], case["E"], case["K"], case["kind"]

    def zeros(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device=DEV)

    if kind == "sort":
        return dict(expert_ids=ids if case["id_bits"] == 64 else ids.to(torch.int32), n_experts=E,
                    order=zeros(N * K, dtype=torch.int32), position=zeros(N, K, dtype=torch.int32),
                    offsets=zeros(E + 1, dtype=torch.int32))
    H, position = case["H"], _positions(ids, E)
    if kind == "dispatch":
        return dict(x=_normal(g, N, H), position=position, out=zeros(N * K, H))
    if kind == "combine":
        return dict(y=_normal(g, N * K, H), position=position, weights=weights if case["weighted"] else None, out=zeros(N, H))
    return dict(dout=_normal(g, N, H), y=_normal(g, N * K, H), position=position, weights=weights, dy=zeros(N * K, H),
                dweights=zeros(N, K, dtype=torch.float32))


def prepare(case, seed):
    args = _attention_inputs(case, seed) if case["kind"] == "attention" else _expert_inputs(case, seed)
    state = dict(kind=case["kind"], args=args)
    if case["kind"] == "attention":
        state["lengths"] = lengths(case)        # a scheduler has them on the host too
    return state


# ---- one pass -------------------------------------------------------------------------------------------------

def run(state):
    kind, args = state["kind"], state["args"]
    if own:
        import paper_2505_11329_amd as tw
        return getattr(tw, {"attention": "attention"}.get(kind, "expert_" + kind))(**args)
    if kind == "attention":
        return _attention(*state["lengths"], **args)
    return {"sort": _sort, "dispatch": _dispatch, "combine": _combine, "combine_backward": _combine_backward}[kind](**args)


PADDED_BYTES = 24 << 30      # of one padded batch's scores


def _attend(q, k, v, q_len, k_len, causal):
    """[B, Lq, Hq, D] and twice [B, Lk, Hk, D], padded; out [B, Lq, Hq, D] and lse [B, Lq, Hq] in fp32."""
    B, Lq, Hq, D = q.shape
    Lk, Hk = k.shape[1:3]
    G = Hq // Hk
    qf = q.float().view(B, Lq, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * Lq, D)
    s = torch.matmul(qf, k.float().permute(0, 2, 3, 1).contiguous()).view(B, Hk, G, Lq, Lk)
    i = torch.arange(Lq, device=q.device)[:, None]
    j = torch.arange(Lk, device=q.device)[None]
    last = k_len[:, None, None] - 1
    if causal:
        last = torch.minimum(last, i + (k_len - q_len)[:, None, None])
    hidden = (j > last)[:, None, None]
    s.mul_(1.0 / math.sqrt(D)).masked_fill_(hidden, -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(B, Hk, G * Lq, Lk), v.float().permute(0, 2, 1, 3).contiguous()).view(B, Hk, G, Lq, D)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (top + total.log()).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(B, Lq, Hq, D), lse.permute(0, 3, 1, 2).reshape(B, Lq, Hq)


def _scattered(like, to, rows):
    """Zeros like `like`, and `rows` in the places `to`; one past the end stands for none."""
    all_ = torch.zeros((like.shape[0] + 1,) + like.shape[1:], dtype=like.dtype, device=like.device)
    all_[to] = rows.to(like.dtype)
    return all_[:-1]


def _rows(offsets, longest, total):
    """Row numbers [B, longest] of the sequences, those past a sequence's end clamped to the tensor."""
    at = offsets[:-1, None].long() + torch.arange(longest, device=offsets.device)
    return at.clamp_(max=total - 1)


def _attention(rows, keys, q, k, v, q_offsets, k_offsets, causal, out, lse):
    B, Lq, Lk = len(rows), max(rows), max(keys)
    q_len, k_len = q_offsets.diff().long(), k_offsets.diff().long()
    if B > 1 and 4 * B * q.shape[1] * Lq * Lk <= PADDED_BYTES:
        # the whole batch at once, padded to its longest sequences
        at = _rows(q_offsets, Lq, q.shape[0])
        from_ = _rows(k_offsets, Lk, k.shape[0])
        o, e = _attend(q[at], k[from_], v[from_], q_len, k_len, causal)
        to = torch.where(torch.arange(Lq, device=q.device) < q_len[:, None], at, q.shape[0])
        return _scattered(out, to, o), _scattered(lse, to, e)
    out, lse = torch.zeros_like(out), torch.zeros_like(lse)
    a = b = 0
    for n, (lq, lk) in enumerate(zip(rows, keys)):
        o, e = _attend(q[None, a:a + lq], k[None, b:b + lk], v[None, b:b + lk], q_len[n:n + 1], k_len[n:n + 1], causal)
        out[a:a + lq], lse[a:a + lq] = o[0].to(out.dtype), e[0]
        a, b = a + lq, b + lk
    return out, lse


def _sort(expert_ids, n_experts, order, position, offsets):
    flat = expert_ids.flatten()
    valid = (flat >= 0) & (flat < n_experts)
    keys, order = torch.sort(torch.where(valid, flat, n_experts), stable=True)
    edges = torch.arange(n_experts + 1, device=flat.device, dtype=keys.dtype)
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=flat.device)
    position = torch.where(valid, place, -1).view(expert_ids.shape)
    return order.to(torch.int32), position.to(torch.int32), torch.searchsorted(keys, edges).to(torch.int32)


def _dispatch(x, position, out):
    to = torch.where(position >= 0, position, out.shape[0]).long()
    return _scattered(out, to, x[:, None].expand(-1, position.shape[1], -1))


def _gathered(y, position):
    """[N, K, H] in fp32, zeros where a pair has no place."""
    has = position >= 0
    return torch.where(has[..., None], y[position.clamp(min=0).long()].float(), 0.0)


def _combine(y, position, weights, out):
    rows = _gathered(y, position)
    return (rows if weights is None else rows * weights[..., None]).sum(1).to(out.dtype)


def _combine_backward(dout, y, position, weights, dy, dweights):
    to = torch.where(position >= 0, position, dy.shape[0]).long()
    d = dout.float()[:, None]
    return _scattered(dy, to, weights[..., None] * d), (_gathered(y, position) * d).sum(-1)


# ---- what a pass cannot do without, and its results in 64 bits --------------------------------------------------

def work(case):
    if case["kind"] == "attention":
        rows, keys = lengths(case)
        Hq, Hk, D = case["heads"], case["kv_heads"], case["dim"]
        pairs = sum(r * k - (r * (r - 1) // 2 if case["causal"] else 0) for r, k in zip(rows, keys))
        return dict(bytes=2 * D * (2 * sum(rows) * Hq + 2 * sum(keys) * Hk) + 4 * sum(rows) * Hq + 8 * (len(rows) + 1),
                    flops=4 * D * Hq * pairs)
    N, K = case["N"], case["K"]
    pairs = (N - case["padded"]) * K
    if case["kind"] == "sort":
        return dict(bytes=N * K * (case["id_bits"] // 8 + 8) + 4 * (case["E"] + 1), flops=N * K)
    H = case["H"]
    if case["kind"] == "dispatch":
        return dict(bytes=2 * H * (N - case["padded"] + pairs) + 4 * N * K, flops=pairs * H)
    if case["kind"] == "combine":
        return dict(bytes=2 * H * (N + pairs) + (8 if case["weighted"] else 4) * N * K, flops=2 * pairs * H)
    return dict(bytes=2 * H * (N - case["padded"] + 2 * pairs) + 12 * N * K, flops=3 * pairs * H)


def exact(case, seed):
    args = prepare(case, seed)["args"]
    if case["kind"] == "attention":
        return _exact_attention(case, **args)
    if case["kind"] == "sort":
        ids, E = args["expert_ids"].cpu().flatten().tolist(), case["E"]
        buckets = [[] for _ in range(E + 1)]
        for p, e in enumerate(ids):
            buckets[e if 0 <= e < E else E].append(p)
        order = [p for b in buckets for p in b]
        offsets, position = [0], [-1] * len(ids)
        for b in buckets[:E]:
            offsets.append(offsets[-1] + len(b))
        for s, p in enumerate(order[:offsets[E]]):
            position[p] = s
        order, position, offsets = (torch.tensor(v, dtype=torch.int32) for v in (order, position, offsets))
        return order, position.view(case["N"], case["K"]), offsets
    position = args["position"].long()
    K = case["K"]
    if case["kind"] == "dispatch":
        out = torch.zeros(args["out"].shape, dtype=torch.float64, device=DEV)
        for k in range(K):
            kept = position[:, k] >= 0
            out[position[kept, k]] = args["x"][kept].double()
        return out
    y = args["y"]
    if case["kind"] == "combine":
        out = torch.zeros(args["out"].shape, dtype=torch.float64, device=DEV)
        for k in range(K):
            kept = position[:, k] >= 0
            w = args["weights"][kept, k, None].double() if case["weighted"] else 1.0
            out[kept] += w * y[position[kept, k]].double()
        return out
    dy = torch.zeros(args["dy"].shape, dtype=torch.float64, device=DEV)
    dweights = torch.zeros(position.shape, dtype=torch.float64, device=DEV)
    for k in range(K):
        kept = position[:, k] >= 0
        d, at = args["dout"][kept].double(), position[kept, k]
        dy[at] = args["weights"][kept, k, None].double() * d
        dweights[kept, k] = (y[at].double() * d).sum(-1)
    return dy, dweights


def _exact_attention(case, q, k, v, q_offsets, k_offsets, causal, out, lse):
    out, lse = torch.zeros(out.shape, dtype=torch.float64, device=DEV), torch.zeros(lse.shape, dtype=torch.float64, device=DEV)
    G = case["heads"] // case["kv_heads"]
    qo, ko = q_offsets.tolist(), k_offsets.tolist()
    for b in range(case["seqs"]):
        lq, lk = qo[b + 1] - qo[b], ko[b + 1] - ko[b]
        seen = None
        if causal:
            seen = torch.ones(lq, lk, dtype=torch.bool, device=DEV).tril(lk - lq)
        for h in range(case["kv_heads"]):
            keys, values = (t[ko[b]:ko[b + 1], h].double() for t in (k, v))
            for head in range(h * G, (h + 1) * G):
                s = q[qo[b]:qo[b + 1], head].double() @ keys.T / math.sqrt(case["dim"])
                if causal:
                    s = torch.where(seen, s, -math.inf)
                e = torch.logsumexp(s, -1)
                lse[qo[b]:qo[b + 1], head] = e
                out[qo[b]:qo[b + 1], head] = torch.exp(s - e[:, None]) @ values
    return out, lse
