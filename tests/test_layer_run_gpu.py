"""A layer's operators as a model with experts runs them: queries and keys normed and rotated in the projection's own rows, then attention;
sort, dispatch, the experts' two products with the gated activation between them, the weighted sum; and a training step's way
back through all of the experts' part and through the norms and the rotation. A padded batch: its last tokens have no position and no
expert. Each operator is held to its 64-bit form on the inputs it met. The same calls in one graph, replayed with other inputs, give
the same bits as eager ones."""
import math

import pytest
import torch

import layer_reference as L
import operator_reference as R

pytestmark = pytest.mark.gpu

EPS = 1e-6


class Model:
    def __init__(self, seed, H, heads, kv_heads, dim, rot, experts, top_k, width, kn):
        g = self.g = torch.Generator().manual_seed(seed)
        self.H, self.heads, self.kv_heads, self.dim, self.experts, self.top_k, self.width, self.kn = H, heads, kv_heads, dim, experts, top_k, width, kn

        def normal(*shape, std=1.0):
            return (std * torch.randn(*shape, generator=g)).bfloat16().cuda()

        self.normal = normal
        self.qkv = normal((heads + 2 * kv_heads) * dim, H, std=H ** -0.5)
        self.q_norm, self.k_norm = 1 + normal(dim, std=0.1), 1 + normal(dim, std=0.1)
        self.rotation = L.table(4096, rot).cuda()
        self.router = normal(experts, H, std=H ** -0.5)
        up, down = (experts, 2 * width, H), (experts, H, width)
        if kn:
            up, down = (experts, H, 2 * width), (experts, width, H)
        self.up, self.down = normal(*up, std=H ** -0.5), normal(*down, std=width ** -0.5)


class Batch:
    """What a step takes: sequences one behind the other, and padding."""

    def __init__(self, m, lengths, padded):
        T = self.T = sum(lengths) + padded
        self.x, self.dout = m.normal(T, m.H), m.normal(T, m.H)
        self.dq, self.dk = m.normal(T, m.heads, m.dim), m.normal(T, m.kv_heads, m.dim)
        self.positions = torch.cat([torch.arange(n) for n in lengths] + [torch.full((padded,), -1)]).cuda()
        self.offsets = R.offsets(lengths).cuda()
        self.live = sum(lengths)
        weights, ids = torch.topk(self.x.float() @ m.router.float().t(), m.top_k, dim=1)
        self.weights, self.ids = torch.softmax(weights, dim=1), torch.where(self.positions[:, None] >= 0, ids, -1)

    def take(self, other):
        for name in ("x", "dout", "dq", "dk", "positions", "offsets", "weights", "ids"):
            getattr(self, name).copy_(getattr(other, name))


def forward(tw, m, b):
    layout = tw.B_KN if m.kn else tw.B_NK
    qkv = tw.gemm_bf16(b.x, m.qkv).view(b.T, -1, m.dim)
    q, k, v = qkv[:, :m.heads], qkv[:, m.heads:m.heads + m.kv_heads], qkv[:, m.heads + m.kv_heads:]
    before = qkv.clone()                                # (the gradient reads what the norms did)
    tw.qk_norm_rope(q, k, b.positions, m.rotation, m.q_norm, m.k_norm, EPS, q_out=q, k_out=k)
    att, lse = tw.attention(q, k, v, b.offsets, b.offsets)
    order, position, offsets = tw.expert_sort(b.ids, m.experts)
    rows = tw.expert_dispatch(b.x, position)
    both = tw.expert_gemm(rows, m.up, offsets, layout)
    h = tw.gated_silu(both, offsets[-1:])
    y = tw.expert_gemm(h, m.down, offsets, layout)
    out = tw.expert_combine(y, position, b.weights)
    return dict(before=before, q=q, k=k, v=v, att=att, lse=lse, weights=b.weights, position=position, offsets=offsets, rows=rows, both=both,
                h=h, y=y, out=out)


def backward(tw, m, b, f):
    layout, other = (tw.B_KN, tw.B_NK) if m.kn else (tw.B_NK, tw.B_KN)
    offsets = f["offsets"]
    dy, dweights = tw.expert_combine_backward(b.dout, f["y"], f["position"], f["weights"])
    dh = tw.expert_gemm(dy, m.down, offsets, other)
    ddown = tw.expert_gemm_backward(f["h"], dy, offsets, layout)
    dboth = tw.gated_silu_backward(dh, f["both"], offsets[-1:])
    drows = tw.expert_gemm(dboth, m.up, offsets, other)
    dup = tw.expert_gemm_backward(f["rows"], dboth, offsets, layout)
    dx = tw.expert_combine(drows, f["position"], None)
    q, k = f["before"][:, :m.heads], f["before"][:, m.heads:m.heads + m.kv_heads]
    dq, dk, dq_norm, dk_norm = tw.qk_norm_rope_backward(b.dq, b.dk, b.positions, m.rotation, q, k, m.q_norm, m.k_norm, EPS)
    return dict(dy=dy, dweights=dweights, dh=dh, ddown=ddown, dboth=dboth, drows=drows, dup=dup, dx=dx, dq=dq, dk=dk, dq_norm=dq_norm, dk_norm=dk_norm)


# one decode-like batch of few rows and ones of more, both layouts of the weights
RUNS = [(dict(H=256, heads=8, kv_heads=2, dim=64, rot=64, experts=16, top_k=2, width=136, kn=False), [1, 3, 1], 2),
        (dict(H=512, heads=4, kv_heads=4, dim=128, rot=128, experts=8, top_k=2, width=264, kn=True), [130, 1, 517, 77], 19),
        (dict(H=520, heads=6, kv_heads=3, dim=80, rot=48, experts=64, top_k=6, width=200, kn=False), [800, 1203], 0)]


@pytest.mark.parametrize("sizes,lengths,padded", RUNS)
def test_forward_and_back(tw, sizes, lengths, padded):
    m = Model(len(lengths), **sizes)
    b = Batch(m, lengths, padded)
    f = forward(tw, m, b)
    live = b.live
    for name, x, weight in (("q", f["before"][:, :m.heads], m.q_norm), ("k", f["before"][:, m.heads:m.heads + m.kv_heads], m.k_norm)):
        want, tol = L.norm_rope(x, weight, b.positions, m.rotation, EPS, False)
        R.assert_close(f[name][:live], want[:live], tol[:live], name)
        assert torch.equal(f[name][live:], x[live:]), name          # padding as the projection left it
    assert torch.equal(f["v"], f["before"][:, m.heads + m.kv_heads:])
    want, want_lse, tol, tol_lse = R.attention(f["q"], f["k"], f["v"], b.offsets, b.offsets, True, 1 / math.sqrt(m.dim))
    R.assert_close(f["att"][:live], want[:live], tol[:live], "attention")
    R.assert_close(f["lse"][:live], want_lse[:live], tol_lse[:live], "lse")
    kept = live * m.top_k
    assert int(f["offsets"][-1]) == kept

    def rows_close(got, pair, what):
        R.assert_close(got[:kept], pair[0][:kept], pair[1][:kept], what)

    rows_close(f["both"], L.product(f["rows"], m.up, f["offsets"], m.kn), "up")
    rows_close(f["h"][:kept], L.gate(f["both"][:kept]), "gate")
    rows_close(f["y"], L.product(f["h"], m.down, f["offsets"], m.kn), "down")
    R.assert_close(f["out"], *R.combine(f["y"], f["position"], f["weights"]), "combine")
    assert not bool(f["out"][live:].any())

    d = backward(tw, m, b, f)
    want, tol, want_w, tol_w = R.combine_backward(b.dout, f["y"], f["position"], f["weights"])
    rows_close(d["dy"], (want, tol), "dy")
    R.assert_close(d["dweights"], want_w, tol_w, "dweights")
    rows_close(d["dh"], L.product(d["dy"], m.down, f["offsets"], not m.kn), "dh")
    R.assert_close(d["ddown"], *L.weight_gradient(f["h"], d["dy"], f["offsets"], m.experts, m.kn), "ddown")
    rows_close(d["dboth"][:kept], L.gate_backward(d["dh"][:kept], f["both"][:kept]), "dboth")
    rows_close(d["drows"], L.product(d["dboth"], m.up, f["offsets"], not m.kn), "drows")
    R.assert_close(d["dup"], *L.weight_gradient(f["rows"], d["dboth"], f["offsets"], m.experts, m.kn), "dup")
    R.assert_close(d["dx"], *R.combine(d["drows"], f["position"], None), "dx")
    assert not bool(d["dx"][live:].any())
    for name, dy, x, weight in (("dq", b.dq, f["before"][:, :m.heads], m.q_norm), ("dk", b.dk, f["before"][:, m.heads:m.heads + m.kv_heads], m.k_norm)):
        want, tol, want_w, tol_w = L.norm_rope_backward(dy, x, weight, b.positions, m.rotation, EPS, False)
        R.assert_close(d[name][:live], want[:live], tol[:live], name)
        R.assert_close(d[name + "_norm"], want_w, tol_w, name + "_norm")


def test_the_experts_gradients_against_those_of_the_whole_expression(tw):
    """dx and the weights' gradients through dispatch, both products, activation and sum, against 64-bit gradients of the expression itself.

    The bound goes the way the values go: what is off so far times the sizes of what it meets, and each step's own rounding to bf16 and
    sum in fp32. With z(g) = g / (1 + exp(-g)): |z'| < 1.1, |z''| <= 1/2, so that z u is off by 1.1 e_g (|u| + e_u) + |z| e_u and its gradients by
    the same rule. The kernels' own fp32 roundings in the activation are less than 2^-20 of values whose gates are below 2^3 here."""
    sizes, lengths, padded = RUNS[1]
    m = Model(5, **sizes)
    b = Batch(m, lengths, padded)
    f = forward(tw, m, b)
    d = backward(tw, m, b, f)
    x, up, down = (t.double().requires_grad_() for t in (b.x, m.up, m.down))
    at, where = f["offsets"].tolist(), f["position"]
    total = torch.zeros(b.T, m.H, dtype=torch.float64, device="cuda")
    off = {"dx": torch.zeros_like(total), "dup": torch.zeros_like(up), "ddown": torch.zeros_like(down)}
    ONE = L.BF16 + 2.0 ** -20

    def times(v, e, w, e_w=0.0):
        """What v w is off by, v and w by e and e_w, rounded to bf16."""
        size = (v.abs() + e) @ (w.abs() + e_w)
        off = size - v.abs() @ w.abs()
        return off + ONE * ((v @ w).abs() + off) + 2 * (v.shape[1] + 1) * L.F32 * size

    assert m.kn
    for e in range(m.experts):
        token, choice = torch.nonzero((where >= at[e]) & (where < at[e + 1]), as_tuple=True)
        weight = f["weights"][token, choice, None].double()
        both = x[token] @ up[e]
        g, u = both.chunk(2, dim=1)
        h = g * torch.sigmoid(g) * u
        total = total.index_add(0, token, weight * (h @ down[e]))
        with torch.no_grad():
            xe, we, te = x[token], up[e], down[e].t().contiguous()
            e_g, e_u = times(xe, 0.0, we).chunk(2, dim=1)
            assert float(g.abs().max()) < 8
            s = torch.sigmoid(g)
            z, dz = (g * s).abs(), (s + g * s * (1 - s)).abs()
            e_h = 1.1 * e_g * (u.abs() + e_u) + z * e_u
            e_h += ONE * (h.abs() + e_h)
            dy = weight * b.dout[token].double()
            e_dy = ONE * dy.abs()
            dh, e_dh = dy @ te, times(dy, e_dy, te)
            e_dg = 1.1 * e_dh * (u.abs() + e_u) + dh.abs() * (dz * e_u + 0.5 * e_g * (u.abs() + e_u))
            e_du = e_dh * (z + 1.1 * e_g) + dh.abs() * 1.1 * e_g
            dboth = torch.cat([dh * u * (s + g * s * (1 - s)), dh * g * s], 1)
            e_dboth = torch.cat([e_dg, e_du], 1)
            e_dboth += ONE * (dboth.abs() + e_dboth)
            rows = dboth @ we.t().contiguous()
            e_rows = times(dboth, e_dboth, we.t().contiguous())
            off["dx"].index_add_(0, token, e_rows + m.top_k * L.F32 * (rows.abs() + e_rows))
            off["dup"][e] = times(xe.t().contiguous(), 0.0, dboth, e_dboth)
            off["ddown"][e] = times(h.t().contiguous(), e_h.t().contiguous(), dy, e_dy)
    (total * b.dout.double()).sum().backward()
    off["dx"] += ONE * (x.grad.abs() + off["dx"])
    for name, want in (("dx", x.grad), ("dup", up.grad), ("ddown", down.grad)):
        R.assert_close(d[name], want, off[name].detach(), name)

@pytest.mark.parametrize("sizes,lengths,padded", RUNS)
def test_captured_and_replayed_with_other_inputs(tw, sizes, lengths, padded):
    m = Model(7, **sizes)
    b = Batch(m, lengths, padded)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            backward(tw, m, b, forward(tw, m, b))
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = forward(tw, m, b)
        d = backward(tw, m, b, f)
    for i in range(3):
        turned = lengths[i % len(lengths):] + lengths[:i % len(lengths)]
        b.take(Batch(m, turned, padded))
        graph.replay()
        torch.cuda.synchronize()
        want_f = forward(tw, m, b)
        want_d = backward(tw, m, b, want_f)
        live, kept = b.live, b.live * m.top_k
        for name, n in (("q", live), ("k", live), ("att", live), ("both", kept), ("h", kept), ("y", kept), ("out", b.T)):
            assert torch.equal(f[name][:n], want_f[name][:n]), (i, name)
        for name, t in d.items():
            n = {"dy": kept, "dh": kept, "dboth": kept, "drows": kept, "dq": live, "dk": live}.get(name, t.shape[0])
            assert torch.equal(t[:n], want_d[name][:n]), (i, name)


def test_more_heads_than_one_launch_takes(tw):
    """2^31 heads of 8 and some: the first tokens, those around where a launch ends, and the last."""
    T, H, D = (1 << 21) + 5, 1024, 8
    g = torch.Generator().manual_seed(9)
    q, k = torch.zeros(T, H, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, 1, D, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 1, 7, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, (1 << 21) - 1, 1 << 21, T - 2, T - 1]).cuda()
    q[rows], k[rows] = (torch.randn(len(rows), n, D, generator=g).bfloat16().cuda() for n in (H, 1))
    rotation, weight = L.table(64, D).cuda(), (1 + 0.1 * torch.randn(D, generator=g)).bfloat16().cuda()
    at = (torch.arange(T, device="cuda", dtype=torch.int32) * 5) % 64
    want = [L.norm_rope(x[rows], weight, at[rows], rotation, EPS, False) for x in (q, k)]
    tw.qk_norm_rope(q, k, at, rotation, weight, weight, EPS, q_out=q, k_out=k)
    R.assert_close(q[rows], *want[0], "q")
    R.assert_close(k[rows], *want[1], "k")
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[rows] = False
    for x in (q, k):        # zeros, of either sign
        assert not bool(x.view(T, -1).amax(1)[keep].any()) and not bool(x.view(T, -1).amin(1)[keep].any())
