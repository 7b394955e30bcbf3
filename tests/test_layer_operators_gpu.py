"""A layer's operators together, as a program has them: fused step, projections, attention, fused step, the experts' products
between sorting and the weighted sum, fused step; unsplit, and in two token splits on two streams, of which the second one's
attention waits for the first one's keys. Each new operator is held to its 64-bit form on the inputs it met, and the split
run to the unsplit one bit for bit. Then the experts' part backwards."""
import math

import pytest
import torch

import operator_reference as R

pytestmark = pytest.mark.gpu

LENGTHS, HEADS, KV_HEADS, DIM, H, EXPERTS, TOP_K, WIDTH = [1700, 2400], 32, 16, 64, 512, 8, 2, 256
CUT = 2600      # inside the second sequence


class Layer:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, std=1.0):
            return (std * torch.randn(*shape, generator=g)).bfloat16().cuda()

        T = sum(LENGTHS)
        self.partials, self.residual = [normal(T, H, std=0.5) for _ in range(2)], normal(T, H)
        self.norms = [1 + normal(H, std=0.1) for _ in range(3)]
        self.qkv = normal((HEADS + 2 * KV_HEADS) * DIM, H, std=H ** -0.5)
        self.o = normal(H, HEADS * DIM, std=(HEADS * DIM) ** -0.5)
        self.router = normal(EXPERTS, H, std=H ** -0.5)
        self.up = [normal(WIDTH, H, std=H ** -0.5) for _ in range(EXPERTS)]
        self.down = [normal(H, WIDTH, std=WIDTH ** -0.5) for _ in range(EXPERTS)]


def attention_rows(a, b):
    """The sequences' parts in rows [a, b): their query rows, and their keys from their first one on."""
    q, k, first_key, at = [], [], None, 0
    for n in LENGTHS:
        lo, hi = max(a, at), min(b, at + n)
        if lo < hi:
            q.append(hi - lo)
            k.append(hi - at)
            first_key = at if first_key is None else first_key
        at += n
    return q, k, first_key


def run(tw, m, a, b, qkv_all, before_attention=None):
    """The layer over rows [a, b) on the current stream; the keys of the whole batch lie in qkv_all."""
    rows = slice(a, b)
    x, res = tw.reduce_add_rmsnorm([p[rows] for p in m.partials], m.residual[rows], m.norms[0], 1e-5)
    tw.gemm_bf16(x, m.qkv, C=qkv_all[rows])
    if before_attention:
        before_attention()
    q_lens, k_lens, first = attention_rows(a, b)
    heads = qkv_all.view(-1, HEADS + 2 * KV_HEADS, DIM)
    q, k, v = heads[rows, :HEADS], heads[first:b, HEADS:HEADS + KV_HEADS], heads[first:b, HEADS + KV_HEADS:]
    qo, ko = R.offsets(q_lens).cuda(), R.offsets(k_lens).cuda()
    att, lse = tw.attention(q, k, v, qo, ko)
    x, res = tw.reduce_add_rmsnorm([tw.gemm_bf16(att.view(b - a, -1), m.o)], res, m.norms[1], 1e-5)
    weights, ids = torch.topk(x.float() @ m.router.float().T, TOP_K, dim=1)
    weights = torch.softmax(weights, dim=1)
    order, position, offsets = tw.expert_sort(ids, EXPERTS)
    at = offsets.tolist()
    rows_in = tw.expert_dispatch(x, position)
    y = torch.empty_like(rows_in)
    for e in range(EXPERTS):
        if at[e] < at[e + 1]:
            here = slice(at[e], at[e + 1])
            tw.gemm_bf16(tw.gemm_bf16(rows_in[here], m.up[e]), m.down[e], C=y[here])
    summed = tw.expert_combine(y, position, weights)
    out, res = tw.reduce_add_rmsnorm([summed], res, m.norms[2], 1e-5)
    return dict(out=out, res=res, summed=summed, y=y, rows_in=rows_in, x=x, position=position, weights=weights, ids=ids, order=order,
                offsets=offsets, att=att, lse=lse, q=q, k=k, v=v, qo=qo, ko=ko)


def test_a_layer_unsplit_and_in_two_splits(tw):
    m, T = Layer(1), sum(LENGTHS)
    sizes = [(len(q), sum(q), b - first) for a, b in ((0, T), (0, CUT), (CUT, T)) for q, _, first in (attention_rows(a, b),)]
    forms = {(f.tile_rows, f.key_waves, f.chunks) for f in (tw.attention_plan(*n, HEADS, KV_HEADS, DIM) for n in sizes)}
    assert len(forms) == 1, forms       # of one form: the same bits
    width = (HEADS + 2 * KV_HEADS) * DIM
    whole = run(tw, m, 0, T, torch.empty(T, width, dtype=torch.bfloat16, device="cuda"))

    # each operator against its 64-bit form
    w = whole
    want, want_lse, tol, tol_lse = R.attention(w["q"], w["k"], w["v"], w["qo"], w["ko"], True, 1 / math.sqrt(DIM))
    R.assert_close(w["att"], want, tol, "attention")
    R.assert_close(w["lse"], want_lse, tol_lse, "lse")
    for name, expected in zip(("order", "position", "offsets"), R.sort(w["ids"], EXPERTS)):
        assert w[name].flatten().tolist() == expected, name
    assert torch.equal(w["rows_in"], w["x"][w["order"].long() // TOP_K])
    R.assert_close(w["summed"], *R.combine(w["y"], w["position"], w["weights"]), "combine")

    # two splits on two streams
    qkv = torch.empty(T, width, dtype=torch.bfloat16, device="cuda")
    here, streams, ready = torch.cuda.current_stream(), [torch.cuda.Stream() for _ in range(2)], torch.cuda.Event()
    parts = []
    for i, (a, b) in enumerate(((0, CUT), (CUT, T))):
        s = streams[i]
        s.wait_stream(here)
        with torch.cuda.stream(s):
            keys_there = (lambda: ready.record(streams[0])) if i == 0 else (lambda: streams[1].wait_event(ready))
            parts.append(run(tw, m, a, b, qkv, keys_there))
    torch.cuda.synchronize()
    for name in ("att", "lse", "summed", "out", "res"):
        assert torch.equal(torch.cat([p[name] for p in parts]), whole[name]), name


def test_the_experts_part_backwards(tw):
    """Gradients of the dispatched rows' products and of the weights, each operator against its 64-bit form, and a token
    whose pairs all have no expert."""
    m = Layer(2)
    g = torch.Generator().manual_seed(3)
    N = 333
    x, up_grad = torch.randn(N, H, generator=g).bfloat16().cuda(), torch.randn(N, H, generator=g).bfloat16().cuda()
    weights, ids = torch.topk(x.float() @ m.router.float().T, TOP_K, dim=1)
    weights = torch.softmax(weights, dim=1)
    ids[7] = -1
    order, position, offsets = tw.expert_sort(ids, EXPERTS)
    at = offsets.tolist()
    rows = tw.expert_dispatch(x, position)
    products = [(m.down[e], slice(at[e], at[e + 1])) for e in range(EXPERTS) if at[e] < at[e + 1]]
    y, drows = torch.zeros(N * TOP_K, WIDTH, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(rows)
    for down, here in products:
        tw.gemm_bf16(rows[here], down, C=y[here], b_layout=tw.B_KN)       # [rows x H] [H x WIDTH]
    up_grad = up_grad[:, :WIDTH].contiguous()
    dy, dw = tw.expert_combine_backward(up_grad, y, position, weights)
    kept = at[EXPERTS]
    want, tol, want_w, tol_w = R.combine_backward(up_grad, y, position, weights)
    R.assert_close(dy[:kept], want[:kept], tol[:kept], "dy")
    R.assert_close(dw, want_w, tol_w, "dweights")
    for down, here in products:
        tw.gemm_bf16(dy[here], down, C=drows[here])                       # [rows x WIDTH] [H x WIDTH]^T
    dx = tw.expert_combine(drows, position)
    R.assert_close(dx, *R.combine(drows, position, None), "dx")
    assert not bool(dx[7].any()) and not bool(dw[7].any())
