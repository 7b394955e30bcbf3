"""What the experts' products, the gated activation and the norms and rotation of queries and keys refuse, without a GPU: every call
here fails its checks before anything could be launched, with addresses that nothing reads."""
import ctypes

import pytest
import torch

import paper_2505_11329_amd as tw
from paper_2505_11329_amd import QkNormRopeArgs

VP = ctypes.c_void_p
OK, E_NULL, E_SHAPE, E_ALIGN, E_ALIAS, E_UNSUP = range(6)
BASE = 0x7000_0000_0000


def addr(i):
    return BASE + i * 0x100_0000


def products(A=addr(0), X=addr(1), out=addr(2), offsets=addr(3), rows=10, N=64, K=128, E=4, layout=0):
    """Both calls: X is B of the one and dC of the other."""
    return tuple(f(VP(A), VP(X), VP(out), VP(offsets), rows, N, K, E, layout, None)
                 for f in (tw.lib().tw_expert_gemm, tw.lib().tw_expert_gemm_backward))


def test_products_refuse():
    for change in (dict(A=None), dict(X=None), dict(out=None), dict(offsets=None)):
        assert products(**change) == (E_NULL,) * 2, change
    for change in (dict(rows=-1), dict(N=-8), dict(K=-8), dict(E=0), dict(E=-1), dict(layout=2), dict(layout=-1)):
        assert products(**change) == (E_SHAPE,) * 2, change
    for change in (dict(rows=1 << 31), dict(N=60), dict(K=4), dict(N=(1 << 17) + 8), dict(K=(1 << 17) + 8), dict(E=1025)):
        assert products(**change) == (E_UNSUP,) * 2, change
    for change in (dict(A=addr(0) + 8), dict(X=addr(1) + 2), dict(out=addr(2) + 4), dict(offsets=addr(3) + 2)):
        assert products(**change) == (E_ALIGN,) * 2, change
    for change in (dict(out=addr(0) + 16), dict(out=addr(1)), dict(out=addr(3) - 16), dict(A=addr(2) + 160)):
        assert products(**change) == (E_ALIAS,) * 2, change
    # nothing to do: nothing is looked at (no rows still leaves gradients of 0 to write)
    assert products(rows=0, A=None, X=None, out=None, offsets=None) == (OK, E_NULL)
    assert products(N=0, A=None, X=None, out=None, offsets=None) == (OK, OK)
    assert products(K=0, out=None)[0] == E_NULL and products(K=0, A=None, X=None, out=None, offsets=None)[1] == OK


def gates(dout=addr(0), x=addr(1), out=addr(2), limit=addr(3), rows=10, F=64):
    return (tw.lib().tw_gated_silu(VP(x), rows, F, VP(limit), VP(out), None),
            tw.lib().tw_gated_silu_backward(VP(dout), VP(x), rows, F, VP(limit), VP(out), None))


def test_gates_refuse():
    for change in (dict(x=None), dict(out=None)):
        assert gates(**change) == (E_NULL,) * 2, change
    assert gates(dout=None)[1] == E_NULL
    for change in (dict(rows=-1), dict(F=0), dict(F=-8)):
        assert gates(**change) == (E_SHAPE,) * 2, change
    for change in (dict(rows=1 << 31), dict(F=60), dict(F=65544)):
        assert gates(**change) == (E_UNSUP,) * 2, change
    for change in (dict(x=addr(1) + 8), dict(out=addr(2) + 2), dict(limit=addr(3) + 2)):
        assert gates(**change) == (E_ALIGN,) * 2, change
    assert gates(dout=addr(0) + 8)[1] == E_ALIGN
    for change in (dict(out=addr(1) + 16), dict(out=addr(3) - 16)):
        assert gates(**change) == (E_ALIAS,) * 2, change
    assert gates(out=addr(1))[0] == E_ALIAS and gates(out=addr(0) + 16)[1] == E_ALIAS and gates(out=addr(0))[1] == E_ALIAS
    assert gates(rows=0, x=None, out=None, dout=None) == (OK,) * 2


def rope_args(**change):
    a = QkNormRopeArgs(q=addr(0), k=addr(1), q_out=addr(2), k_out=addr(3), positions=addr(4), rotation=addr(5), q_weight=addr(6),
                       k_weight=addr(7), tokens=10, n_positions=100, q_stride=512, k_stride=128, q_out_stride=512, k_out_stride=128,
                       position_bytes=8, q_heads=8, kv_heads=2, head_dim=64, rot_dim=64, interleaved=0, eps=1e-6, dq=addr(8), dk=addr(9),
                       dq_weight=addr(10), dk_weight=addr(11), dq_stride=512, dk_stride=128)
    for name, value in change.items():
        setattr(a, name, value)
    return a


def rope(workspace=addr(12), size=1 << 20, **change):
    a = rope_args(**change)
    return (tw.lib().tw_qk_norm_rope(ctypes.byref(a), None),
            tw.lib().tw_qk_norm_rope_backward(ctypes.byref(a), VP(workspace), size, None))


def test_norm_rope_refuses():
    assert tw.lib().tw_qk_norm_rope(None, None) == E_NULL and tw.lib().tw_qk_norm_rope_backward(None, None, 0, None) == E_NULL
    for change in (dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(positions=None), dict(rotation=None),
                   dict(q_weight=None), dict(k_weight=None), dict(q_weight=None, k_weight=None, rotation=None, positions=None)):
        assert rope(**change) == (E_NULL,) * 2, change
    for change in (dict(dq=None), dict(dk=None), dict(dq_weight=None), dict(dk_weight=None)):
        assert rope(**change)[1] == E_NULL, change
    for change in (dict(tokens=-1), dict(q_heads=0), dict(kv_heads=0), dict(head_dim=0), dict(n_positions=-1), dict(rot_dim=0),
                   dict(rot_dim=72), dict(q_stride=504), dict(k_stride=120), dict(q_out_stride=-512), dict(k_out_stride=0), dict(eps=-1.0),
                   dict(eps=float("nan")), dict(eps=float("inf"))):
        assert rope(**change) == (E_SHAPE,) * 2, change
    for change in (dict(dq_stride=504), dict(dk_stride=0)):
        assert rope(**change)[1] == E_SHAPE, change
    for change in (dict(tokens=1 << 31), dict(head_dim=60), dict(head_dim=136), dict(q_heads=1025), dict(kv_heads=1025), dict(rot_dim=20),
                   dict(n_positions=1 << 31), dict(position_bytes=2), dict(q_stride=516), dict(k_out_stride=(1 << 22) + 8)):
        assert rope(**change) == (E_UNSUP,) * 2, change
    for change in (dict(q=addr(0) + 8), dict(k=addr(1) + 2), dict(q_out=addr(2) + 8), dict(k_out=addr(3) + 4), dict(positions=addr(4) + 4),
                   dict(rotation=addr(5) + 8), dict(q_weight=addr(6) + 2), dict(k_weight=addr(7) + 8)):
        assert rope(**change) == (E_ALIGN,) * 2, change
    for change in (dict(dq=addr(8) + 8), dict(dk=addr(9) + 2), dict(dq_weight=addr(10) + 2), dict(dk_weight=addr(11) + 1)):
        assert rope(**change)[1] == E_ALIGN, change
    # outputs over inputs, other columns, tables and each other
    for change in (dict(q_out=addr(1)), dict(k_out=addr(0)), dict(k_out=addr(2)), dict(q_out=addr(0) + 16), dict(q_out=addr(0), q_out_stride=520),
                   dict(k_out=addr(4)), dict(q_out=addr(5) + 1024), dict(k_out=addr(6)), dict(q_out=addr(7) - 64)):
        assert rope(**change) == (E_ALIAS,) * 2, change
    for change in (dict(q_out=addr(8) + 16), dict(k_out=addr(8)), dict(q_out=addr(10)), dict(dq_weight=addr(11)), dict(dk_weight=addr(0)),
                   dict(dq_weight=addr(6)), dict(dk_weight=addr(9) + 64)):
        assert rope(**change)[1] == E_ALIAS, change
    # one buffer of 1024 columns: columns that cross the row's end or meet
    wide = dict(q_stride=1024, k_stride=1024, q_out_stride=1024, k_out_stride=1024, q=addr(0), k=addr(0) + 1024, k_out=addr(0) + 1024)
    assert rope(**wide, q_out=addr(0) + 1008) == (E_ALIAS,) * 2                     # its end in the keys' columns
    assert rope(**wide, q_out=addr(0) + 1280) == (E_ALIAS,) * 2                     # its end in the next row's queries
    need = tw.qk_norm_rope_backward_workspace_bytes(10, 8, 2, 64, 64)
    assert need > 0 and need % (64 * 4) == 0        # rows of 64 sums, for the queries and for the keys
    assert rope(workspace=None)[1] == E_NULL and rope(size=need - 1)[1] == E_SHAPE and rope(workspace=addr(12) + 8)[1] == E_ALIGN
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11):
        assert rope(workspace=addr(i), size=need)[1] == E_ALIAS, i
    # nothing to do: nothing is looked at, but the weights' gradients are written
    nothing = dict(tokens=0, q=None, k=None, q_out=None, k_out=None, positions=None, dq=None, dk=None)
    assert rope(**nothing, q_weight=None, k_weight=None) == (OK, OK)
    assert rope(**nothing, dq_weight=None) == (OK, E_NULL) and rope(**nothing, dk_weight=addr(10) + 16) == (OK, E_ALIAS)


def test_norm_rope_workspace():
    f = tw.lib().tw_qk_norm_rope_backward_workspace_bytes
    assert f(None) == -1 and f(ctypes.byref(rope_args(head_dim=60))) == -1 and f(ctypes.byref(rope_args(tokens=0))) == 0
    assert f(ctypes.byref(rope_args(q_weight=None))) == 0
    assert f(ctypes.byref(rope_args())) == tw.qk_norm_rope_backward_workspace_bytes(10, 8, 2, 64, 64)
    assert 0 < tw.qk_norm_rope_backward_workspace_bytes(1 << 30, 8, 2, 128) <= 1 << 24


def test_the_binding_refuses_tensors_in_host_memory_and_wrong_shapes():
    x, i32 = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32)
    for call, name in ((lambda: tw.expert_gemm(x, x, i32), "A"), (lambda: tw.expert_gemm_backward(x, x, i32), "A"),
                       (lambda: tw.gated_silu(x), "x"), (lambda: tw.gated_silu_backward(x, x), "x"),
                       (lambda: tw.qk_norm_rope(x, x, i32, x), "q"), (lambda: tw.qk_norm_rope_backward(x, x, i32, x), "dq")):
        with pytest.raises(TypeError, match=name + " must be a GPU tensor"):
            call()


@pytest.mark.gpu
def test_the_binding_refuses_wrong_tensors_on_the_gpu():
    def bf16(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")

    A, B, at = bf16(6, 64), bf16(3, 32, 64), torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad, message in ((lambda: tw.expert_gemm(A, bf16(3, 32, 72), at), "B has shape"), (lambda: tw.expert_gemm(A, B, at[:3]), "offsets has shape"),
                         (lambda: tw.expert_gemm(A, B, at, 2), "b_layout"), (lambda: tw.expert_gemm(A[:, :32], bf16(3, 32, 32), at), "contiguous"),
                         (lambda: tw.expert_gemm(A, B, at, C=bf16(6, 64)), "C has shape"), (lambda: tw.expert_gemm(A, A, at), "B must be"),
                         (lambda: tw.expert_gemm_backward(A, bf16(5, 32), at), "dC has shape"),
                         (lambda: tw.expert_gemm_backward(A, bf16(6, 32), at, dB=bf16(3, 64, 32)), "dB has shape"),
                         (lambda: tw.gated_silu(bf16(3, 33)), "2F"), (lambda: tw.gated_silu(A, at), "limit has shape"),
                         (lambda: tw.gated_silu_backward(A, A), "dout has shape")):
        with pytest.raises(ValueError, match=message):
            bad()
    with pytest.raises(TypeError, match="offsets must be int32"):
        tw.expert_gemm(A, B, at.long())
    with pytest.raises(TypeError, match="B must be bfloat16"):
        tw.expert_gemm(A, B.float(), at)
    q, k, p, r, w = bf16(4, 8, 64), bf16(4, 2, 64), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(9, 64, device="cuda"), bf16(64)
    for bad, message in ((lambda: tw.qk_norm_rope(q, bf16(5, 2, 64), p, r), "k has shape"), (lambda: tw.qk_norm_rope(q, k, p[:3], r), "positions has"),
                         (lambda: tw.qk_norm_rope(q, k, None, r), "belong together"), (lambda: tw.qk_norm_rope(q, k, p, r, w), "belong together"),
                         (lambda: tw.qk_norm_rope(q, k, p, torch.zeros(9, 72, device="cuda")), "more columns"),
                         (lambda: tw.qk_norm_rope(q, k, p, r[:0]), "rotation must be"), (lambda: tw.qk_norm_rope(q, k, p, r, w, w[:32]), "k_weight has"),
                         (lambda: tw.qk_norm_rope(q[..., ::2], k[..., ::2], p, r[:, :32].contiguous()), "next to each other"),
                         (lambda: tw.qk_norm_rope_backward(q, k, p, r, q[:3], k, w, w), "q has shape")):
        with pytest.raises(ValueError, match=message):
            bad()
    with pytest.raises(TypeError, match="positions must be int32 or int64"):
        tw.qk_norm_rope(q, k, p.float(), r)
    with pytest.raises(TypeError, match="q must be a GPU tensor"):
        tw.qk_norm_rope_backward(q, k, p, r, q_weight=w, k_weight=w)
    with pytest.raises(tw.TwError):
        tw.qk_norm_rope(q, k, None, None)


def test_norm_rope_workspace_before_the_tensors_are_there():
    """Whether there is a rotation yet does not change the size: what the query says suffices for the call with one and without."""
    f = tw.lib().tw_qk_norm_rope_backward_workspace_bytes
    for tokens, q_heads, kv_heads, dim in ((1, 1, 1, 8), (10, 8, 2, 64), (40, 8, 2, 128), (300, 28, 4, 72), (20000, 32, 8, 128)):
        for rot in range(8, dim + 1, 8):
            for interleaved in (0, 1):
                sizes = dict(tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, head_dim=dim, rot_dim=rot, interleaved=interleaved,
                             q_stride=q_heads * dim, k_stride=kv_heads * dim, q_out_stride=q_heads * dim, k_out_stride=kv_heads * dim,
                             dq_stride=q_heads * dim, dk_stride=kv_heads * dim)
                for i, name in enumerate(("q", "k", "q_out", "k_out", "dq", "dk")):
                    sizes[name] = BASE + (i + 1) * 0x10_0000_0000
                none = dict(rotation=None, positions=None)
                need = f(ctypes.byref(rope_args(**{**sizes, **none})))
                assert need > 0 and need == f(ctypes.byref(rope_args(**sizes))), sizes
                bare = QkNormRopeArgs(tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, head_dim=dim, rot_dim=rot, interleaved=interleaved,
                                      q_weight=16, position_bytes=4)
                assert f(ctypes.byref(bare)) == need, sizes
                # enough (the address is refused after the size), and with the rotation not more than it takes
                for given in ({}, none):
                    a = rope_args(**{**sizes, **given})
                    assert tw.lib().tw_qk_norm_rope_backward(ctypes.byref(a), VP(addr(12) + 8), need, None) == E_ALIGN, (sizes, given)
                a = rope_args(**sizes)
                assert tw.lib().tw_qk_norm_rope_backward(ctypes.byref(a), VP(addr(12)), need - 1, None) == E_SHAPE, sizes
    # a rot_dim that is none where there is no rotation does not count
    for rot in (0, -8, 20, 72, 1 << 30):
        assert f(ctypes.byref(rope_args(rotation=None, positions=None, rot_dim=rot))) == tw.qk_norm_rope_backward_workspace_bytes(10, 8, 2, 64)


def test_expert_gemm_plan():
    L, launch = tw.lib(), tw.ExpertGemmLaunch()

    def plan(rows=10, N=64, K=128, E=4, layout=0, backward=0, cus=256, to=ctypes.byref(launch)):
        return L.tw_expert_gemm_plan(rows, N, K, E, layout, backward, cus, to)

    for backward in (0, 1):
        assert plan(backward=backward, to=None) == E_NULL
        for change in (dict(rows=-1), dict(N=-8), dict(K=-8), dict(E=0), dict(layout=2), dict(cus=0), dict(cus=-1)):
            assert plan(backward=backward, **change) == E_SHAPE, change
        for change in (dict(rows=1 << 31), dict(N=60), dict(K=4), dict(N=(1 << 17) + 8), dict(K=(1 << 17) + 8), dict(E=1025)):
            assert plan(backward=backward, **change) == E_UNSUP, change
        assert plan(backward=backward, N=0) == OK and launch.tiles == launch.workgroups == launch.tile_rows == launch.tile_cols == 0
    assert plan(rows=0) == OK and launch.tiles == 0
    assert plan(rows=0, backward=1) == OK and launch.tiles > 0      # gradients of 0 are written
    assert plan(K=0) == OK and launch.tiles > 0                     # and sums of nothing
    assert plan(K=0, backward=1) == OK and launch.tiles == 0
    for layout in (0, 1):
        # no more tiles than a launch takes, whatever the sizes; as many workgroups as compute units for tiles that fill one
        for rows in (1, 7, 100, 5000, 100_000, (1 << 31) - 1):
            for E in (1, 8, 1024):
                for N, K in ((8, 8), (4096, 2048), (1 << 17, 64), (1 << 17, 1 << 17)):
                    if rows * N >= 1 << 46:     # more than 2^30 tiles: results of 140 TB
                        continue
                    f = tw.expert_gemm_plan(rows, N, K, E, layout)
                    assert 1 <= f.tiles <= 1 << 30 and f.tile_rows >= 16 and f.tile_cols >= 32, (rows, E, N, K)
                    assert f.tiles >= (rows + f.tile_rows - 1) // f.tile_rows * ((N + f.tile_cols - 1) // f.tile_cols)
                    assert f.workgroups == 256 if f.tile_rows == 256 and f.tiles > 256 else f.tiles <= f.workgroups < f.tiles + 8
                    b = tw.expert_gemm_plan(rows, N, K, E, layout, True)
                    edge = b.tile_rows
                    assert edge == b.tile_cols and edge in (128, 256) and b.tiles == -(-N // edge) * -(-K // edge) * E and b.workgroups >= 1
