"""The gated activation and the norms and rotation of queries and keys at sizes that one launch does not take, or whose heads 32 bits do
not count: rows that repeat, so that what the first of them give is what all do."""
import pytest
import torch

import layer_reference as L
import operator_reference as R

pytestmark = pytest.mark.gpu


def normal(g, *shape):
    return torch.randn(*shape, generator=g).bfloat16().cuda()


def repeated(base, rows):
    return base.repeat(-(-rows // base.shape[0]), *[1] * (base.dim() - 1))[:rows]


def all_rows_are(got, base):
    whole = got.shape[0] // base.shape[0]
    part = 1 << 10
    for i in range(0, whole, part):
        n = min(part, whole - i)
        if not bool((got[i * base.shape[0]:(i + n) * base.shape[0]].view(n, *base.shape) == base).all()):
            return False
    rest = got.shape[0] - whole * base.shape[0]
    return torch.equal(got[whole * base.shape[0]:], base[:rest])


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def test_gate_of_more_than_2_30_pieces(tw):
    rows, period = (1 << 30) + 77, 4099
    g = torch.Generator().manual_seed(1)
    base, d_base = normal(g, period, 16), normal(g, period, 8)
    want, d_want = tw.gated_silu(base), tw.gated_silu_backward(d_base, base)
    R.assert_close(want, *L.gate(base), "gate")
    R.assert_close(d_want, *L.gate_backward(d_base, base), "gradient")
    x, limit = repeated(base, rows), torch.tensor([rows - 20], dtype=torch.int32, device="cuda")
    out = torch.full((rows, 8), 7.0, dtype=torch.bfloat16, device="cuda")
    tw.gated_silu(x, limit, out=out)
    assert all_rows_are(out[:rows - 20], want) and bool((out[rows - 20:] == 7.0).all())
    del out
    last = x[rows - 20:].clone()
    tw.gated_silu_backward(repeated(d_base, rows), x, limit, dx=x)
    assert all_rows_are(x[:rows - 20], d_want) and torch.equal(x[rows - 20:], last)


@pytest.mark.parametrize("dim,rot,interleaved", [(8, 8, False), (128, 128, True)])
def test_rotation_of_more_heads_than_a_launch_takes(tw, dim, rot, interleaved):
    """2^22 workgroups of 256 heads of 8, or of 32 heads of 128."""
    heads, period = 1024, 1031
    tokens = (1 << 22) * (256 if dim == 8 else 32) // heads + 5
    g = torch.Generator().manual_seed(dim)
    q_base, k_base, rotation, w = normal(g, period, heads, dim), normal(g, period, 1, dim), L.table(100, rot).cuda(), normal(g, dim)
    at_base = torch.randint(-3, 100, (period,), generator=g).cuda()
    want = [t.clone() for t in (q_base, k_base)]
    tw.qk_norm_rope(q_base, k_base, at_base, rotation, w, w, interleaved=interleaved, q_out=want[0], k_out=want[1])
    has = at_base >= 0
    for x, out in zip((q_base, k_base), want):
        R.assert_close(out[has], *(t[has] for t in L.norm_rope(x, w, at_base, rotation, 1e-6, interleaved)), "rotation")
        assert torch.equal(out[~has], x[~has])
    q, k, at = repeated(q_base, tokens), repeated(k_base, tokens), repeated(at_base, tokens)
    tw.qk_norm_rope(q, k, at, rotation, w, w, interleaved=interleaved, q_out=q, k_out=k)
    assert all_rows_are(q, want[0]) and all_rows_are(k, want[1])


def test_gradient_of_more_than_2_32_heads(tw):
    heads, dim, period = 1024, 8, 1031
    tokens = (1 << 22) + 3
    assert tokens * heads > 1 << 32
    g = torch.Generator().manual_seed(3)
    q_base, k_base, rotation = normal(g, period, heads, dim), normal(g, period, 1, dim), L.table(100, dim).cuda()
    at_base = torch.randint(0, 100, (period,), generator=g).cuda()
    want = tw.qk_norm_rope_backward(q_base, k_base, at_base, rotation)
    for x, out in zip((q_base, k_base), want):
        R.assert_close(out, *L.norm_rope_backward(x, None, None, at_base, rotation, 0.0, False)[:2], "gradient")
    q, k, at = repeated(q_base, tokens), repeated(k_base, tokens), repeated(at_base, tokens)
    tw.qk_norm_rope_backward(q, k, at, rotation, dq_out=q, dk_out=k)
    assert all_rows_are(q, want[0]) and all_rows_are(k, want[1])
