"""Tokens sorted by expert, copied to their places, summed back, and the gradient: against plain 64-bit forms."""
import math

import pytest
import torch

import operator_reference as R
from helpers import captured_kernels

pytestmark = pytest.mark.gpu


def ids_of(N, K, E, seed=0, none=0.1, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, E, (N, K), generator=g)
    drop = torch.rand(N, K, generator=g) < none
    ids[drop] = torch.tensor([-1, E, 1 << 30])[torch.randint(0, 3, (int(drop.sum()),), generator=g)]
    return ids.to(dtype).cuda()


def routed(N, K, E, H, seed=0, none=0.1):
    g = torch.Generator().manual_seed(seed + 1000)
    _, position, _ = R.sort(ids_of(N, K, E, seed, none), E)
    position = torch.tensor(position, dtype=torch.int32).view(N, K).cuda()

    def normal(*shape):
        return torch.randn(*shape, generator=g).bfloat16().cuda()

    return position, normal(N, H), normal(N * K, H), torch.rand(N, K, generator=g).cuda()


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("N,K,E", [(0, 2, 8), (1, 1, 1), (3, 2, 8), (64, 6, 64), (77, 8, 160), (1023, 4, 512), (1024, 4, 513), (1025, 4, 1024),
                                   (2047, 4, 8), (2048, 4, 16), (5000, 8, 128), (16384, 8, 256), (9, 32, 40)])
def test_sort(tw, N, K, E, dtype):
    for none in (0.0, 0.15, 1.0):
        print(N, K, E, dtype, none, flush=True)
        ids = ids_of(N, K, E, seed=N, none=none, dtype=dtype)
        got = [t.flatten().tolist() for t in tw.expert_sort(ids, E)]
        for name, x, y in zip(("order", "position", "offsets"), got, R.sort(ids, E)):
            assert x == y, name


def test_sort_ids_far_outside_and_all_the_same(tw):
    for fill in (5, -(1 << 63), (1 << 63) - 1, (1 << 32) + 5, 7):
        ids = torch.full((3000, 3), fill, dtype=torch.int64, device="cuda")
        ids[17, 1] = 2
        for x, y in zip(tw.expert_sort(ids, 8), R.sort(ids, 8)):
            assert x.flatten().tolist() == y


SIZES = [(1, 1, 4, 8), (5, 2, 4, 64), (33, 3, 8, 520), (64, 8, 16, 2048), (17, 11, 32, 2056), (100, 6, 64, 5120), (3, 32, 64, 16384), (2, 2, 2, 65536)]


@pytest.mark.parametrize("N,K,E,H", SIZES)
def test_dispatch(tw, N, K, E, H):
    position, x, _, _ = routed(N, K, E, H)
    out = torch.full((N * K, H), 7.0, dtype=torch.bfloat16, device="cuda")
    want = out.clone()
    for k in range(K):
        has = position[:, k] >= 0
        want[position[has, k].long()] = x[has]
    assert tw.expert_dispatch(x, position, out=out) is out and torch.equal(out, want)


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("N,K,E,H", SIZES)
def test_combine(tw, N, K, E, H, weighted):
    position, _, y, w = routed(N, K, E, H)
    w = w if weighted else None
    want, tol = R.combine(y, position, w)
    R.assert_close(tw.expert_combine(y, position, w), want, tol, "combine")


@pytest.mark.parametrize("weighted", [True, False])
def test_combine_into_more_than_the_caches_keep(tw, weighted):
    N, K, H = 4400, 2, 16384
    position, _, y, w = routed(N, K, 8, H)
    assert N * H * 2 > 128 << 20
    w = w if weighted else None
    want, tol = R.combine(y, position, w)
    R.assert_close(tw.expert_combine(y, position, w), want, tol, "combine")


@pytest.mark.parametrize("N,K,E,H", SIZES)
def test_combine_backward(tw, N, K, E, H):
    position, dout, y, w = routed(N, K, E, H)
    dy = torch.full_like(y, math.nan)
    _, dw = tw.expert_combine_backward(dout, y, position, w, dy=dy)
    want, tol, want_w, tol_w = R.combine_backward(dout, y, position, w)
    R.assert_close(dy, want, tol, "dy")         # rows that no pair has: NaN as before
    R.assert_close(dw, want_w, tol_w, "dweights")
    in_place = y.clone()
    _, dw2 = tw.expert_combine_backward(dout, in_place, position, w, dy=in_place)
    assert torch.equal(dw, dw2)
    has = torch.unique(position[position >= 0]).long()
    assert torch.equal(in_place[has], dy[has])


@pytest.mark.parametrize("N,K,E,H", [(1400, 3, 16, 2056),      # two pairs to a workgroup, the last of them alone
                                     (2100, 4, 8, 8192)])      # more than the caches keep
def test_many_rows_out_and_back(tw, N, K, E, H):
    position, x, y, w = routed(N, K, E, H)
    dy = torch.full_like(y, math.nan)
    _, dw = tw.expert_combine_backward(x, y, position, w, dy=dy)
    want, tol, want_w, tol_w = R.combine_backward(x, y, position, w)
    R.assert_close(dy, want, tol, "dy")
    R.assert_close(dw, want_w, tol_w, "dweights")
    out = torch.zeros_like(y)
    tw.expert_dispatch(x, position, out=out)
    has = position >= 0
    assert torch.equal(out[position[has].long()], x[:, None].expand(N, K, H)[has])
    assert int((out != 0).any(dim=1).sum()) == int(has.sum())


def test_gradients_against_differences(tw):
    """Both are gradients of sums that are linear in each argument: central differences in 64 bits are exact but for
    rounding (values below 2^6 and steps of 1: 2^-40 at most)."""
    N, K, E, H = 4, 3, 4, 16
    position, x, y, w = routed(N, K, E, H, seed=3)
    g = torch.Generator().manual_seed(5)
    up, up_rows = torch.randn(N, H, generator=g).bfloat16().cuda(), torch.randn(N * K, H, generator=g).bfloat16().cuda()
    dy, dw = tw.expert_combine_backward(up, y, position, w)

    def total(y_, w_):
        return float((R.combine(y_, position, w_)[0] * up.double()).sum())

    for row, col in ((0, 0), (3, 7), (5, 15)):
        step = torch.zeros(y.shape, dtype=torch.float64, device="cuda")
        step[row, col] = 1.0
        slope = (total(y.double() + step, w.double()) - total(y.double() - step, w.double())) / 2
        assert abs(float(dy[row, col]) - slope) <= R.BF16 * abs(slope) + 2.0 ** -22
    for n in range(N):
        for k in range(K):
            step = torch.zeros(w.shape, dtype=torch.float64, device="cuda")
            step[n, k] = 1.0
            slope = (total(y.double(), w.double() + step) - total(y.double(), w.double() - step)) / 2
            assert abs(float(dw[n, k]) - slope) <= H * R.F32 * 64
    # dispatch: its gradient is the unweighted sum
    dx = tw.expert_combine(up_rows, position)
    for n, col in ((0, 0), (2, 9)):
        places = [int(s) for s in position[n] if s >= 0]
        slope = sum(float(up_rows[s, col].double()) for s in places)       # each place is a copy of x[n]
        assert abs(float(dx[n, col]) - slope) <= R.BF16 * abs(slope) + 2.0 ** -22


def test_values_and_weights_of_pairs_without_a_place_have_no_part(tw):
    N, K, E, H = 40, 4, 8, 256
    position, dout, y, w = routed(N, K, E, H, none=0.4)
    out = tw.expert_combine(y, position, w)
    dy, dw = tw.expert_combine_backward(dout, y, position, w, dy=torch.zeros_like(y))
    kept = int((position >= 0).sum())
    y2, w2 = y.clone(), torch.where(position < 0, math.nan, w)
    y2[kept:] = math.nan
    assert torch.equal(tw.expert_combine(y2, position, w2), out)
    dy2, dw2 = tw.expert_combine_backward(dout, y2, position, w2, dy=torch.zeros_like(y))
    assert torch.equal(dy2, dy) and torch.equal(dw2, dw)
    # places outside the rows there are: none
    few = y[:kept // 2].contiguous()
    cut = torch.where(position < kept // 2, position, -1)
    assert torch.equal(tw.expert_combine(few, position, w), tw.expert_combine(few, cut, w))
    out = torch.zeros_like(few)
    tw.expert_dispatch(dout, position, out=out)
    assert torch.equal(out, tw.expert_dispatch(dout, cut, out=torch.zeros_like(few)))
    # a token without any pair: exactly 0
    none = torch.full_like(position, -1)
    assert not bool(tw.expert_combine(y2, none, w2).any())
    assert not bool(tw.expert_combine_backward(dout, y2, none, w2)[1].any())
    # special values go through where they are seen
    y3 = y.clone()
    y3[0, 3], y3[1, 4] = math.inf, math.nan
    got, (want, tol) = tw.expert_combine(y3, position, w), R.combine(y3, position, w)
    R.assert_close(got, want, torch.nan_to_num(tol, 0.0, 0.0, 0.0), "Inf and NaN")


def test_rows_beyond_32_bit_offsets(tw):
    H, rows = 16384, 140000         # 4.3 GiB
    y = torch.empty(rows, H, dtype=torch.bfloat16, device="cuda")
    position = torch.tensor([[rows - 1, 5], [-1, rows - 2]], dtype=torch.int32, device="cuda")
    x = torch.randn(2, H, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    tw.expert_dispatch(x, position, out=y)
    assert torch.equal(y[rows - 1], x[0]) and torch.equal(y[5], x[0]) and torch.equal(y[rows - 2], x[1])
    w = torch.tensor([[0.5, 0.25], [1.0, 2.0]], device="cuda")
    R.assert_close(tw.expert_combine(y, position, w), *R.combine(y, position, w), "combine")
    tw.expert_combine_backward(x, y, position, w, dy=y)
    assert torch.equal(y[rows - 1], x[0] * 0.5) and torch.equal(y[rows - 2], x[1] * 2)


def test_streams_and_graphs(tw):
    """The four calls on a side stream, and captured, replayed with other inputs among eager calls."""
    N, K, E, H = 700, 8, 64, 512
    ids = [ids_of(N, K, E, seed=s) for s in (1, 2)]
    g = torch.Generator().manual_seed(0)
    x, w = torch.randn(N, H, generator=g).bfloat16().cuda(), torch.rand(N, K, generator=g).cuda()

    def step(i, **more):
        order, position, offsets = tw.expert_sort(i, E, **more)
        rows = tw.expert_dispatch(x, position, out=torch.zeros(N * K, H, dtype=torch.bfloat16, device="cuda"), **more)
        out = tw.expert_combine(rows, position, w, **more)
        dy, dw = tw.expert_combine_backward(x, rows, position, w, dy=torch.zeros_like(rows), **more)
        return order, position, offsets, rows, out, dy, dw

    want = [step(i) for i in ids]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for i, e in zip(ids, want):
            for a, b in zip(step(i, stream=side), e):
                assert torch.equal(a, b)
    torch.cuda.synchronize()
    held = ids[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(held)
    for n in range(4):
        held.copy_(ids[n % 2])
        graph.replay()
        eager = step(ids[(n + 1) % 2])
        torch.cuda.synchronize()
        for a, b in zip(got, want[n % 2]):
            assert torch.equal(a, b)
        for a, b in zip(eager, want[(n + 1) % 2]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("N,K,H", [(64, 8, 4096), (1000, 2, 2048)])
def test_room_to_spare_changes_nothing(tw, N, K, H):
    """A buffer with more rows than there are pairs: the launch is that of one that fits, since it writes as much."""
    position, x, y, w = routed(N, K, 16, H)
    many = (160 << 20) // (H * 2)
    results = []
    for rows in (N * K, many):
        out, y2 = torch.zeros(rows, H, dtype=torch.bfloat16, device="cuda"), torch.zeros(rows, H, dtype=torch.bfloat16, device="cuda")
        y2[:N * K] = y
        dy, dw, s = torch.zeros_like(y2), torch.zeros_like(w), torch.cuda.Stream()
        torch.cuda.synchronize()
        kernels = captured_kernels(s, lambda: (tw.expert_dispatch(x, position, out=out, stream=s),
                                               tw.expert_combine_backward(x, y2, position, w, dy=dy, dweights=dw, stream=s)))
        assert len(kernels) == 2
        tw.expert_dispatch(x, position, out=out)
        tw.expert_combine_backward(x, y2, position, w, dy=dy, dweights=dw)
        assert not bool(out[N * K:].any()) and not bool(dy[N * K:].any())
        results.append((kernels, out[:N * K], dy[:N * K], dw))
    assert results[0][0] == results[1][0]
    for a, b in zip(results[0][1:], results[1][1:]):
        assert torch.equal(a, b)
