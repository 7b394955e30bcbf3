"""What tw_attention and the experts' calls refuse, without a GPU: every call here fails its checks before anything could
be launched, with addresses that nothing reads."""
import ctypes

import pytest
import torch

import paper_2505_11329_amd as tw
from paper_2505_11329_amd.binding import AttentionArgs, AttentionLaunch

VP = ctypes.c_void_p
OK, E_NULL, E_SHAPE, E_ALIGN, E_ALIAS, E_UNSUP = range(6)
BASE = 0x7000_0000_0000


def addr(i):
    return BASE + i * 0x100_0000


def attention(workspace=None, workspace_bytes=0, **change):
    """A call that is right but for `change`, and has no workspace where it needs some."""
    a = AttentionArgs(q=addr(0), k=addr(1), v=addr(2), out=addr(3), lse=addr(4), q_offsets=addr(5), k_offsets=addr(6), n_seqs=2,
                      q_rows=2, k_rows=9000, q_stride=512, k_stride=128, v_stride=128, out_stride=512, q_heads=8, kv_heads=2,
                      head_dim=64, scale=0.125, causal=1)
    for name, value in change.items():
        setattr(a, name, value)
    return tw.lib().tw_attention(ctypes.byref(a), VP(workspace), workspace_bytes, VP(None))


def test_attention_refuses():
    assert tw.lib().tw_attention(None, None, 0, None) == E_NULL
    for name in ("q", "k", "v", "out", "q_offsets", "k_offsets"):
        assert attention(**{name: None}) == E_NULL, name
    for name in ("q", "k", "v", "out"):
        assert attention(**{name: addr(7) + 8}) == E_ALIGN, name
    for name in ("lse", "q_offsets", "k_offsets"):
        assert attention(**{name: addr(7) + 2}) == E_ALIGN, name
    for change in (dict(n_seqs=-1), dict(q_rows=-1), dict(k_rows=-1), dict(q_heads=0), dict(kv_heads=0), dict(kv_heads=3),
                   dict(kv_heads=16), dict(head_dim=0), dict(q_stride=504), dict(k_stride=120), dict(v_stride=0),
                   dict(out_stride=-512), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan"))):
        assert attention(**change) == E_SHAPE, change
    for change in (dict(head_dim=60), dict(head_dim=136, q_stride=2048, k_stride=512, v_stride=512, out_stride=2048),
                   dict(q_stride=516), dict(k_stride=(1 << 22) + 8), dict(q_heads=1026, q_stride=1 << 17, out_stride=1 << 17),
                   dict(n_seqs=(1 << 14) + 1), dict(q_rows=1 << 31), dict(k_rows=1 << 31), dict(q_rows=1 << 29),
                   dict(q_rows=1 << 29, q_heads=2, q_stride=128, out_stride=128)):
        assert attention(**change) == E_UNSUP, change
    need = 2 * 8 * 66 * 4 * plan(2, 2, 9000, 8, 2, 64).chunks
    assert attention() == E_NULL                                    # no workspace
    assert attention(addr(8), need - 1) == E_SHAPE
    assert attention(addr(8) + 8, need) == E_ALIGN
    assert attention(addr(3), need) == E_ALIAS                      # is out
    assert attention(addr(1), need) == E_ALIAS                      # is k
    for change in (dict(out=addr(0)), dict(out=addr(0) + 1024), dict(out=addr(1) + 16), dict(out=addr(2) + 9000 * 256 - 16),
                   dict(out=addr(5)), dict(lse=addr(3)), dict(lse=addr(6)), dict(lse=addr(1))):
        assert attention(addr(8), need, **change) == E_ALIAS, change
    # nothing to do: nothing is looked at
    assert attention(n_seqs=0, q=None, out=None, q_offsets=None) == OK
    assert attention(q_rows=0, q=None, out=None) == OK


def test_attention_refuses_scales():
    for scale in (0.0, -1.0, 3.0e38, float("inf"), float("nan")):
        assert attention(scale=scale) == E_SHAPE, scale
    assert attention(scale=1.7e38, n_seqs=0) == OK


def plan(*sizes):
    return tw.attention_plan(*sizes)


def test_attention_plan_and_workspace():
    L = tw.lib()
    assert L.tw_attention_plan(None, ctypes.byref(AttentionLaunch())) == E_NULL
    assert L.tw_attention_workspace_bytes(None) == -1
    with pytest.raises(tw.TwError):
        plan(1, 1, 1, 8, 3, 64)
    assert plan(0, 5, 5, 8, 2, 64).chunks == 0 and tw.attention_workspace_bytes(0, 5, 5, 8, 2, 64) == 0
    for sizes in ((1, 1, 1, 8, 2, 64), (48, 48, 200000, 64, 8, 128), (1, 100, 9000, 16, 2, 128), (1, 4096, 16384, 64, 8, 128),
                  (64, 64, 64, 1, 1, 8), (1, 1, 0, 4, 4, 64), (1 << 14, 1 << 14, 1 << 30, 8, 1, 128)):
        f = plan(*sizes)
        assert f.chunks >= 1 and f.min_chunk >= 128 and f.tile_rows > 0
        assert tw.attention_workspace_bytes(*sizes) == (0 if f.chunks == 1 else f.chunks * sizes[1] * sizes[3] * (sizes[5] + 2) * 4)
    assert tw.attention_workspace_bytes(1, 1, 1, 8, 3, 64) == -1


def sort(ids=addr(0), id_bytes=4, N=10, top_k=2, E=8, order=addr(1), position=addr(2), offsets=addr(3), workspace=None, size=0):
    return tw.lib().tw_expert_sort(VP(ids), id_bytes, N, top_k, E, VP(order), VP(position), VP(offsets), VP(workspace), size, None)


def test_expert_sort_refuses():
    for change in (dict(ids=None), dict(order=None), dict(position=None), dict(offsets=None), dict(N=1 << 20)):
        assert sort(**change) == E_NULL, change
    assert sort(N=0, offsets=None) == E_NULL
    for change in (dict(N=-1), dict(top_k=0), dict(E=0), dict(E=-1)):
        assert sort(**change) == E_SHAPE, change
    for change in (dict(E=1025), dict(top_k=33), dict(N=1 << 30), dict(id_bytes=2), dict(id_bytes=0)):
        assert sort(**change) == E_UNSUP, change
    for change in (dict(ids=addr(0) + 2), dict(ids=addr(0) + 4, id_bytes=8), dict(order=addr(1) + 1), dict(position=addr(1) + 2),
                   dict(offsets=addr(1) + 3)):
        assert sort(**change) == E_ALIGN, change
    need = tw.expert_sort_workspace_bytes(1 << 16, 2, 8)
    assert need > 0 and need % (9 * 4) == 0
    assert sort(N=1 << 16, workspace=addr(4), size=need - 1) == E_SHAPE
    assert sort(N=1 << 16, workspace=addr(4) + 2, size=need) == E_ALIGN
    for change in (dict(order=addr(0)), dict(position=addr(1) + 76), dict(offsets=addr(2) + 4), dict(offsets=addr(0) - 4)):
        assert sort(**change) == E_ALIAS, change
    assert sort(N=1 << 16, workspace=addr(1), size=need) == E_ALIAS
    assert tw.expert_sort_workspace_bytes(10, 2, 8) == 0 and tw.expert_sort_workspace_bytes(10, 2, 0) == -1


def rows_calls(N=10, top_k=2, H=64, rows=20, a=addr(0), b=addr(1), position=addr(2), weights=addr(3), out=addr(4), out_w=addr(5)):
    """The three calls over rows: a [N x H] (or, summed, rows x H), b the rows that the gradient reads."""
    L = tw.lib()
    return (L.tw_expert_dispatch(VP(a), VP(position), N, top_k, H, VP(out), rows, None),
            L.tw_expert_combine(VP(a), rows, VP(position), VP(weights), N, top_k, H, VP(out), None),
            L.tw_expert_combine_backward(VP(a), VP(b), rows, VP(position), VP(weights), N, top_k, H, VP(out), VP(out_w), None))


def test_expert_rows_refuse():
    for change in (dict(a=None), dict(position=None), dict(out=None)):
        assert rows_calls(**change) == (E_NULL,) * 3, change
    for change in (dict(b=None), dict(weights=None, a=None), dict(out_w=None)):
        assert rows_calls(**change)[2] == E_NULL, change
    for change in (dict(N=-1), dict(top_k=0), dict(H=0), dict(H=-8), dict(rows=-1)):
        assert rows_calls(**change) == (E_SHAPE,) * 3, change
    for change in (dict(top_k=33), dict(N=1 << 30), dict(H=60), dict(H=65544), dict(rows=1 << 31)):
        assert rows_calls(**change) == (E_UNSUP,) * 3, change
    for change in (dict(a=addr(0) + 8), dict(position=addr(2) + 2), dict(out=addr(4) + 4)):
        assert rows_calls(**change) == (E_ALIGN,) * 3, change
    assert rows_calls(weights=addr(3) + 1)[1:] == (E_ALIGN,) * 2
    for change in (dict(b=addr(1) + 2), dict(out_w=addr(5) + 2)):
        assert rows_calls(**change)[2] == E_ALIGN, change
    for change in (dict(out=addr(0) + 128), dict(out=addr(2)), dict(a=addr(4))):
        assert rows_calls(**change) == (E_ALIAS,) * 3, change
    assert rows_calls(out=addr(3))[1:] == (E_ALIAS,) * 2
    for change in (dict(out=addr(1) + 128), dict(out_w=addr(0)), dict(out_w=addr(1)), dict(out_w=addr(3)), dict(out_w=addr(4) + 16)):
        assert rows_calls(**change)[2] == E_ALIAS, change
    assert rows_calls(N=0, a=None, position=None, out=None, b=None, weights=None, out_w=None) == (OK,) * 3


def test_the_binding_refuses_tensors_in_host_memory_and_wrong_shapes():
    x, i32 = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(TypeError, match="q must be a GPU tensor"):
        tw.attention(x.view(4, 1, 64), x, x, i32, i32)
    with pytest.raises(TypeError, match="expert_ids must be a GPU tensor"):
        tw.expert_sort(i32, 8)
    with pytest.raises(TypeError, match="x must be a GPU tensor"):
        tw.expert_dispatch(x, i32)
    with pytest.raises(TypeError, match="y must be a GPU tensor"):
        tw.expert_combine(x, i32)
    with pytest.raises(TypeError, match="y must be a GPU tensor"):
        tw.expert_combine_backward(x, None, i32, None)
