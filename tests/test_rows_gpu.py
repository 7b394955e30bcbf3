"""The gated activation, and the norms and rotation of queries and keys, with their gradients, against plain 64-bit forms."""
import math

import pytest
import torch

import layer_reference as L
import operator_reference as R

pytestmark = pytest.mark.gpu


def normal(g, *shape, std=1.0):
    return (std * torch.randn(*shape, generator=g)).bfloat16().cuda()


def nans(*shape):
    return torch.full(shape, math.nan, dtype=torch.bfloat16, device="cuda")


# ---- gated activation ----

@pytest.mark.parametrize("rows,F", [(1, 8), (3, 24), (7, 1408), (64, 2048), (333, 520), (1000, 4096), (2, 65536), (9000, 8192)])
def test_gate(tw, rows, F):
    g = torch.Generator().manual_seed(rows)
    x, dout = normal(g, rows, 2 * F, std=3.0), normal(g, rows, F)
    x[0, :4] = torch.tensor([0.0, 88.0, -88.0, 200.0])
    out = nans(rows, F)
    assert tw.gated_silu(x, out=out) is out
    R.assert_close(out, *L.gate(x), "gate")
    dx = tw.gated_silu_backward(dout, x)
    R.assert_close(dx, *L.gate_backward(dout, x), "gradient")
    in_place = x.clone()
    assert tw.gated_silu_backward(dout, in_place, dx=in_place) is in_place and torch.equal(in_place, dx)


@pytest.mark.parametrize("limit", [-3, 0, 1, 50, 99, 100, 5000])
def test_gate_leaves_rows_behind_the_limit(tw, limit):
    g = torch.Generator().manual_seed(2)
    rows, F = 100, 136
    x, dout, live = normal(g, rows, 2 * F), normal(g, rows, F), min(max(limit, 0), rows)
    x[live:], dout[live:] = math.inf, math.nan
    at = torch.tensor([limit], dtype=torch.int32, device="cuda")
    out = tw.gated_silu(x, at, out=nans(rows, F))
    dx = tw.gated_silu_backward(dout, x, at, dx=nans(rows, 2 * F))
    assert bool(out[live:].isnan().all()) and bool(dx[live:].isnan().all())
    R.assert_close(out[:live], *L.gate(x[:live]), "gate")
    R.assert_close(dx[:live], *L.gate_backward(dout[:live], x[:live]), "gradient")


def test_gate_of_large_and_infinite_values(tw):
    """Every bf16 as a gate: finite ones give what the formula gives, Inf and NaN propagate and stay in their element."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).cuda()
    x = torch.cat([bits.view(-1, 64), torch.full((1024, 64), 1.5, dtype=torch.bfloat16, device="cuda")], 1)
    out = tw.gated_silu(x)
    finite = bits.view(-1, 64).isfinite()
    want, tol = L.gate(torch.where(torch.cat([finite, finite], 1), x, 1.0))
    over = want.abs() > 3.38e38      # rounds to Inf, or next to it
    R.assert_close(torch.where(finite & ~over, out, 0.0), torch.where(finite & ~over, want, 0.0), tol, "gate")
    special = bits.view(-1, 64)
    assert bool((out[special == math.inf] == math.inf).all()) and bool(out[special.isnan()].isnan().all())
    assert not bool(out[finite & ~over].isnan().any())


def test_gate_gradient_against_differences(tw):
    g = torch.Generator().manual_seed(4)
    x, dout = normal(g, 4, 48, std=2.0), normal(g, 4, 24)
    dx = tw.gated_silu_backward(dout, x).double().cpu()
    at, d = x.double().cpu(), dout.double().cpu()

    def loss(t):
        return (t[:, :24] * torch.sigmoid(t[:, :24]) * t[:, 24:] * d).sum()

    h = 1e-5    # third derivatives below 2^5 here: h^2 of that, and 2^-52 of the sum over h
    for i in range(4):
        for j in range(48):
            up, down = at.clone(), at.clone()
            up[i, j] += h
            down[i, j] -= h
            want = float(loss(up) - loss(down)) / (2 * h)
            assert abs(float(dx[i, j]) - want) <= (L.BF16 + 1e-5) * abs(want) + 1e-6, (i, j)


# ---- norms and rotation ----

def heads(g, T, Hq, Hk, D, packed, std=1.0):
    """Queries and keys, as columns of a projection's output or on their own."""
    if packed:
        qkv = normal(g, T, Hq + 2 * Hk, D, std=std)
        return qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv
    return normal(g, T, Hq, D, std=std), normal(g, T, Hk, D, std=std), None


def positions(g, T, most, dtype, padding=0.1):
    p = torch.randint(0, most, (T,), generator=g)
    drop = torch.rand(T, generator=g) < padding
    wrong = [-1, most, (1 << 31) - 1] + ([-(1 << 62), 1 << 32] if dtype == torch.int64 else [])
    p[drop] = torch.tensor(wrong)[torch.randint(0, len(wrong), (int(drop.sum()),), generator=g)]
    return p.to(dtype).cuda()


# tokens, q_heads, kv_heads, dim, rot (0: none), interleaved, norm
CASES = [(1, 1, 1, 8, 8, False, True), (1, 8, 2, 64, 64, False, True), (2, 3, 1, 16, 16, True, True), (5, 16, 2, 72, 72, False, True),
         (9, 16, 2, 72, 72, True, True), (48, 64, 8, 128, 128, False, True), (33, 24, 8, 80, 80, False, True), (17, 20, 20, 96, 96, True, True),
         (21, 20, 20, 96, 48, False, True), (40, 12, 4, 128, 32, False, True), (40, 12, 4, 128, 40, False, True), (40, 12, 4, 128, 64, True, True),
         (100, 8, 2, 64, 64, False, False), (100, 7, 3, 40, 24, False, False), (100, 7, 3, 40, 24, True, False), (64, 8, 1, 128, 0, False, True),
         (30, 5, 5, 24, 0, True, True), (700, 28, 4, 128, 128, False, True), (3001, 32, 8, 128, 128, False, True), (4000, 16, 16, 64, 64, True, True),
         (9, 1024, 1, 8, 8, False, True), (2500, 64, 8, 128, 96, False, False), (3, 1, 1024, 128, 104, False, True)]


def make(case, seed=0, dtype=torch.int64, packed=True, most=500, eps=1e-6):
    T, Hq, Hk, D, rot, interleaved, norm = case
    g = torch.Generator().manual_seed(seed + T + D)
    q, k, qkv = heads(g, T, Hq, Hk, D, packed)
    at = positions(g, T, most, dtype) if rot else None
    rotation = L.table(most, rot).cuda() if rot else None
    w = [(1 + 0.2 * torch.randn(D, generator=g)).bfloat16().cuda() if norm else None for _ in range(2)]
    return g, q, k, qkv, at, rotation, w, dict(eps=eps, interleaved=interleaved)


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("case", CASES)
def test_norm_rope(tw, case, packed):
    T, Hq, Hk, D = case[:4]
    for dtype in (torch.int32, torch.int64):
        _, q, k, qkv, at, rotation, w, more = make(case, dtype=dtype, packed=packed)
        q_out, k_out = nans(T, Hq, D), nans(T, Hk, D)
        got = tw.qk_norm_rope(q, k, at, rotation, *w, **more, q_out=q_out, k_out=k_out)
        assert got[0] is q_out and got[1] is k_out
        for name, out, x, weight in (("q", q_out, q, w[0]), ("k", k_out, k, w[1])):
            R.assert_close(out, *L.norm_rope(x, weight, at, rotation, more["eps"], more["interleaved"]), name)
    # in place: the same bits, padding and the values' columns as they were
    if packed:
        was, has = qkv.clone(), ~q_out.isnan().all(2).all(1)
        tw.qk_norm_rope(q, k, at, rotation, *w, **more, q_out=q, k_out=k)
        assert torch.equal(q[has], q_out[has]) and torch.equal(k[has], k_out[has])
        assert torch.equal(qkv[~has], was[~has]) and torch.equal(qkv[:, Hq + Hk:], was[:, Hq + Hk:])


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("case", CASES)
def test_norm_rope_backward(tw, case, packed):
    T, Hq, Hk, D = case[:4]
    g, q, k, _, at, rotation, w, more = make(case, packed=packed)
    dq, dk, _ = heads(g, T, Hq, Hk, D, packed)
    norm = case[6]
    dq_out, dk_out = nans(T, Hq, D), nans(T, Hk, D)
    given = dict(q=q, k=k, q_weight=w[0], k_weight=w[1]) if norm else {}
    got = tw.qk_norm_rope_backward(dq, dk, at, rotation, **given, **more, dq_out=dq_out, dk_out=dk_out)
    for name, out, dw, dy, x, weight in (("q", got[0], got[2], dq, q, w[0]), ("k", got[1], got[3], dk, k, w[1])):
        want, tol, want_w, tol_w = L.norm_rope_backward(dy, x, weight, at, rotation, more["eps"], more["interleaved"])
        R.assert_close(out, want, tol, "d" + name)
        if norm:
            R.assert_close(dw, want_w, tol_w, "dweight of " + name)
        else:
            assert dw is None
    # over the gradients that came in, and over the inputs
    has = ~dq_out.isnan().all(2).all(1)
    for over in ("gradients", "inputs"):
        dq2, dk2, args = dq.clone(), dk.clone(), {n: t.clone() for n, t in given.items()}
        if over == "inputs" and not norm:
            continue
        to = (dq2, dk2) if over == "gradients" else (args["q"], args["k"])
        got2 = tw.qk_norm_rope_backward(dq2, dk2, at, rotation, **args, **more, dq_out=to[0], dk_out=to[1])
        assert torch.equal(to[0][has], dq_out[has]) and torch.equal(to[1][has], dk_out[has]), over
        if norm:
            assert torch.equal(got2[2], got[2]) and torch.equal(got2[3], got[3]), over


def test_positions_far_out(tw):
    """A table of a million positions, its last rows used."""
    T, most = 40, 1 << 20
    g = torch.Generator().manual_seed(3)
    q, k = normal(g, T, 4, 128), normal(g, T, 2, 128)
    rotation = L.table(most, 128, base=5e5).cuda()
    at = (most - 1 - torch.arange(T) * 7).cuda()
    for x, out in zip((q, k), tw.qk_norm_rope(q, k, at, rotation)):
        R.assert_close(out, *L.norm_rope(x, None, at, rotation, 0.0, False), "far")


def test_rows_beyond_4_gib(tw):
    T, stride = 600, 1 << 22
    assert (T - 1) * stride * 2 > 1 << 32
    buffer = torch.zeros(T, stride, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(11)
    values = normal(g, T, 6 * 64)
    buffer[:, :384] = values
    q, k = buffer[:, :256].unflatten(1, (4, 64)), buffer[:, 256:384].unflatten(1, (2, 64))
    rotation, w = L.table(T, 64).cuda(), normal(g, 64)
    at = torch.arange(T, device="cuda")
    want = [L.norm_rope(x.clone(), w, at, rotation, 1e-6, False) for x in (q, k)]
    tw.qk_norm_rope(q, k, at, rotation, w, w, q_out=q, k_out=k)
    R.assert_close(q, *want[0], "q")
    R.assert_close(k, *want[1], "k")


def test_norms_of_zeros_large_and_infinite_heads(tw):
    """A head of zeros is 0 with eps > 0; Inf and NaN stay in their head; eps counts for small ones."""
    g = torch.Generator().manual_seed(4)
    q, k = normal(g, 6, 4, 64), normal(g, 6, 2, 64)
    q[0, 0], q[1, 1], q[2, 2, 5], q[3, 3, 7], k[4, 0], k[5] = 0, 1e-4, math.inf, math.nan, 1e18, 1e-20
    w = [normal(g, 64) for _ in range(2)]
    rotation, at = L.table(16, 64).cuda(), torch.arange(6).cuda()
    out = tw.qk_norm_rope(q, k, at, rotation, *w)
    for x, weight, got in zip((q, k), w, out):
        clean = torch.where(x.isfinite().all(2, keepdim=True), x, 1.0)
        want, tol = L.norm_rope(clean, weight, at, rotation, 1e-6, False)
        bad = ~x.isfinite().all(2)
        R.assert_close(torch.where(bad[..., None], 0.0, got), torch.where(bad[..., None], 0.0, want), tol, "finite heads")
    # x / Inf is 0 and Inf / Inf NaN; of pairs with the NaN both
    assert bool(out[0][2, 2, [5, 37]].isnan().all()) and bool(out[0][3, 3].isnan().all())
    # without norms an infinite value reaches its pair only
    plain = tw.qk_norm_rope(q, k, at, rotation)
    assert int((~plain[0][2, 2].isfinite()).sum()) == 2


def test_gradients_against_differences(tw):
    T, Hq, Hk, D = 3, 2, 1, 16
    for rot, interleaved in ((16, False), (8, True), (8, False)):
        g, q, k, _, _, rotation, w, more = make((T, Hq, Hk, D, rot, interleaved, True), packed=False, eps=1e-3)
        at = torch.tensor([3, 77, 401]).cuda()
        dq, dk = normal(g, T, Hq, D), normal(g, T, Hk, D)
        got = tw.qk_norm_rope_backward(dq, dk, at, rotation, q, k, *w, **more)
        _, cos, sin = L._angles(at.cpu(), rotation.cpu())

        def loss(x, weight, dy):
            z = x / torch.sqrt(x.square().mean(2, keepdim=True) + more["eps"]) * weight
            return (L.turned(z, cos, sin, interleaved) * dy).sum()

        h = 1e-5
        for x, weight, dy, dx, dw in ((q, w[0], dq, got[0], got[2]), (k, w[1], dk, got[1], got[3])):
            x, weight, dy = x.double().cpu(), weight.double().cpu(), dy.double().cpu()
            for t, grad, rounding in ((x, dx, L.BF16), (weight, dw, 1e-5)):
                for i in range(0, t.numel(), 3):
                    moved = []
                    for step in (h, -h):
                        u = t.clone()
                        u.view(-1)[i] += step
                        moved.append(loss(u, weight, dy) if t is x else loss(x, u, dy))
                    want = float(moved[0] - moved[1]) / (2 * h)
                    # (1e-5: fp32 sums of up to 16 x 6 terms around 1, and of the difference itself)
                    assert abs(float(grad.view(-1)[i]) - want) <= rounding * abs(want) + 1e-4, (rot, interleaved, i)


def test_captured_calls(tw):
    """Forward and backward in one graph, with other inputs and positions at each replay, eager work in between."""
    for case in ((7, 8, 2, 128, 128, False, True), (1500, 16, 4, 64, 64, False, True)):
        T, Hq, Hk, D = case[:4]
        g, q, k, _, at, rotation, w, more = make(case, packed=False)
        dq, dk = normal(g, T, Hq, D), normal(g, T, Hk, D)
        room = torch.empty(tw.qk_norm_rope_backward_workspace_bytes(T, Hq, Hk, D, D), dtype=torch.uint8, device="cuda")
        out = [torch.zeros_like(t) for t in (q, k, dq, dk)]
        dw = [torch.zeros(D, device="cuda") for _ in range(2)]
        x, h = normal(g, T, 64), torch.zeros(T, 32, dtype=torch.bfloat16, device="cuda")

        def calls():
            tw.qk_norm_rope(q, k, at, rotation, *w, **more, q_out=out[0], k_out=out[1])
            tw.qk_norm_rope_backward(dq, dk, at, rotation, q, k, *w, **more, dq_out=out[2], dk_out=out[3], dq_weight=dw[0],
                                     dk_weight=dw[1], workspace=room)
            tw.gated_silu(x, out=h)

        calls()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for i in range(4):
            for t in (q, k, dq, dk, x):
                t.copy_(normal(g, *t.shape))
            at.copy_(positions(g, T, 500, at.dtype))
            for t in out + dw:
                t.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            want = [torch.full_like(t, 3.0) for t in out]
            tw.qk_norm_rope(q, k, at, rotation, *w, **more, q_out=want[0], k_out=want[1])
            want_w = tw.qk_norm_rope_backward(dq, dk, at, rotation, q, k, *w, **more, dq_out=want[2], dk_out=want[3])[2:]
            for a, b in zip(out + dw + [h], want + list(want_w) + [tw.gated_silu(x)]):
                assert torch.equal(a, b), i


def test_no_tokens(tw):
    g, q, k, _, at, rotation, w, more = make((0, 4, 2, 64, 64, False, True), packed=False)
    assert tw.qk_norm_rope(q, k, at, rotation, *w, **more)[0].shape == (0, 4, 64)
    got = tw.qk_norm_rope_backward(q, k, at, rotation, q, k, *w, **more)
    assert not bool(got[2].any()) and not bool(got[3].any())
    at = torch.full((5,), -1, device="cuda")            # nothing but padding
    dq, dk = nans(5, 4, 64), nans(5, 2, 64)
    got = tw.qk_norm_rope_backward(normal(g, 5, 4, 64), normal(g, 5, 2, 64), at, rotation, normal(g, 5, 4, 64), normal(g, 5, 2, 64), *w, **more,
                                   dq_out=dq, dk_out=dk)
    assert bool(dq.isnan().all()) and not bool(got[2].any()) and not bool(got[3].any())
    assert tw.gated_silu(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")).shape == (0, 32)


def test_heads_whose_squares_overflow_are_0(tw):
    """The sum of squares is in fp32: Inf from 2^128 on. Other heads of the token are as they are without it."""
    g = torch.Generator().manual_seed(6)
    q, k = normal(g, 5, 4, 64), normal(g, 5, 2, 64)
    w, rotation, at = normal(g, 64), L.table(16, 64).cuda(), torch.arange(5).cuda()
    clean = tw.qk_norm_rope(q, k, at, rotation, w, w)
    q[1, 2, 7], k[3, 1] = -2.0 ** 64, 2.0 ** 62
    out = tw.qk_norm_rope(q, k, at, rotation, w, w)
    assert not bool(out[0][1, 2].any()) and not bool(out[1][3, 1].any())
    for x, was, head in ((out[0], clean[0], (1, 2)), (out[1], clean[1], (3, 1))):
        x[head] = was[head]
        assert torch.equal(x, was)
