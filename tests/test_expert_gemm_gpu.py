"""The experts' products and the gradient of their weights against plain 64-bit forms."""
import math

import pytest
import torch

import layer_reference as L
import operator_reference as R

pytestmark = pytest.mark.gpu


def normal(g, *shape, std=1.0):
    return (std * torch.randn(*shape, generator=g)).bfloat16().cuda()


def weights(g, E, N, K, kn, std=None):
    shape = (E, K, N) if kn else (E, N, K)
    return normal(g, *shape, std=K ** -0.5 if std is None else std)


def counted(g, rows, E, ahead=0, behind=0):
    """Offsets of E experts over all but the first and last rows, some of them without any."""
    cuts = sorted(torch.randint(ahead, rows - behind + 1, (E - 1,), generator=g).tolist())
    return torch.tensor([ahead] + cuts + [rows - behind], dtype=torch.int32).cuda()


def check(tw, A, B, offsets, kn, what="C"):
    C = torch.full((A.shape[0], B.shape[2 if kn else 1]), math.nan, dtype=torch.bfloat16, device="cuda")
    assert tw.expert_gemm(A, B, offsets, tw.B_KN if kn else tw.B_NK, C=C) is C
    R.assert_close(C, *L.product(A, B, offsets, kn), what)      # rows without an expert: NaN as before
    return C


def check_gradient(tw, A, dC, offsets, E, kn):
    dB = tw.expert_gemm_backward(A, dC, offsets, tw.B_KN if kn else tw.B_NK)
    R.assert_close(dB, *L.weight_gradient(A, dC, offsets, E, kn), "dB")
    return dB


SIZES = [  # rows, E, N, K
    (1, 1, 8, 8), (1, 4, 16, 40), (3, 8, 64, 64), (17, 3, 72, 136), (64, 1, 64, 256), (65, 2, 136, 512), (130, 70, 48, 24),
    (257, 5, 264, 1000), (300, 16, 128, 520), (511, 8, 520, 72), (640, 2, 256, 264), (1000, 130, 64, 128), (1500, 3, 776, 640),
    (2100, 4, 512, 520), (900, 1024, 24, 32), (3, 1, 4104, 2056), (40, 4, 2048, 4096), (48, 2, 1000, 7168)]


@pytest.mark.parametrize("kn", [False, True])
@pytest.mark.parametrize("rows,E,N,K", SIZES)
def test_products(tw, rows, E, N, K, kn):
    g = torch.Generator().manual_seed(rows + E)
    A, B = normal(g, rows, K), weights(g, E, N, K, kn)
    for ahead, behind in ((0, 0), (min(rows, 1), 0), (0, rows // 3), (rows // 2, rows - rows // 2)):
        print(rows, E, N, K, kn, ahead, behind, flush=True)
        check(tw, A, B, counted(g, rows, E, ahead, behind), kn)


@pytest.mark.parametrize("kn", [False, True])
@pytest.mark.parametrize("rows,E,N,K", SIZES)
def test_weight_gradients(tw, rows, E, N, K, kn):
    g = torch.Generator().manual_seed(rows + E)
    A, dC = normal(g, rows, K), normal(g, rows, N)
    for ahead, behind in ((0, 0), (min(rows, 1), 0), (0, rows // 3), (rows // 2, rows - rows // 2)):
        print(rows, E, N, K, kn, ahead, behind, flush=True)
        check_gradient(tw, A, dC, counted(g, rows, E, ahead, behind), E, kn)


def exact_inputs(g, *shape):
    """Small whole numbers: every sum of them is exact in fp32, whatever its order."""
    return torch.randint(-3, 4, shape, generator=g).to(torch.bfloat16).cuda()


# one expert with most rows, some with a few, at sizes of every form of the launch
EXACT = [([2, 0, 1, 5], 64, 520), ([16, 3, 1, 16], 1000, 1032), ([40, 17, 0, 33], 264, 2048), ([100, 64, 65, 63], 320, 192),
         ([300, 1, 256, 129], 392, 328), ([1025, 511, 0, 7], 512, 1096), ([2000, 2048, 100, 1500], 1160, 840),
         ([5000, 3, 700], 776, 1544), ([9, 11, 8, 12] * 32, 136, 1024)]


@pytest.mark.parametrize("kn", [False, True])
@pytest.mark.parametrize("lengths,N,K", EXACT)
def test_products_of_whole_numbers_are_exact(tw, lengths, N, K, kn):
    """Sums below 2^24 are exact, and their one rounding is to the nearest: equal to the last bit."""
    g = torch.Generator().manual_seed(len(lengths))
    E, rows = len(lengths), sum(lengths) + 5
    A, offsets = exact_inputs(g, rows, K), R.offsets(lengths, 2).cuda()
    B = exact_inputs(g, *((E, K, N) if kn else (E, N, K)))
    C = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    want = C.clone()
    for e, lo, hi in L.rows_of(offsets, rows):
        want[lo:hi] = (A[lo:hi].float() @ (B[e].float() if kn else B[e].float().t())).bfloat16()
    assert torch.equal(tw.expert_gemm(A, B, offsets, int(kn), C=C), want)


@pytest.mark.parametrize("kn", [False, True])
@pytest.mark.parametrize("lengths,N,K", EXACT)
def test_weight_gradients_of_whole_numbers_are_exact(tw, lengths, N, K, kn):
    g = torch.Generator().manual_seed(len(lengths))
    E, rows = len(lengths), sum(lengths) + 5
    A, dC, offsets = exact_inputs(g, rows, K), exact_inputs(g, rows, N), R.offsets(lengths, 2).cuda()
    want = torch.zeros((E, K, N) if kn else (E, N, K), dtype=torch.bfloat16, device="cuda")
    for e, lo, hi in L.rows_of(offsets, rows):
        x, d = A[lo:hi].float(), dC[lo:hi].float()
        want[e] = (x.t() @ d if kn else d.t() @ x).bfloat16()
    dB = torch.full_like(want, math.nan)
    assert torch.equal(tw.expert_gemm_backward(A, dC, offsets, int(kn), dB=dB), want)


def test_nothing_to_multiply(tw):
    g = torch.Generator().manual_seed(1)
    none = torch.zeros(5, dtype=torch.int32, device="cuda")
    assert tw.expert_gemm(normal(g, 0, 64), weights(g, 4, 32, 64, False), none).shape == (0, 32)
    assert not bool(tw.expert_gemm_backward(normal(g, 0, 64), normal(g, 0, 32), none).any())
    A, B = normal(g, 9, 64), weights(g, 4, 32, 64, False)
    check(tw, A, B, none, False)                                            # no expert has a row
    assert not bool(check_gradient(tw, A, normal(g, 9, 32), none, 4, False).any())
    C = torch.full((9, 32), 5.0, dtype=torch.bfloat16, device="cuda")       # sums of nothing
    tw.expert_gemm(normal(g, 9, 0), torch.empty(4, 32, 0, dtype=torch.bfloat16, device="cuda"), R.offsets([3, 0, 2, 1], 1).cuda(), C=C)
    assert not bool(C[1:7].any()) and bool((C[:1] == 5).all()) and bool((C[7:] == 5).all())


@pytest.mark.parametrize("rows,N,K", [(40, 72, 136), (700, 520, 264)])
@pytest.mark.parametrize("kn", [False, True])
def test_infinite_values_stay_in_their_row_and_expert(tw, rows, N, K, kn):
    """NaN in rows of other experts, and in rows of none, meets no other row's sums; nor do other experts' weights."""
    g = torch.Generator().manual_seed(5)
    E = 4
    A, dC, B = normal(g, rows, K), normal(g, rows, N), weights(g, E, N, K, kn)
    third = rows // 3
    offsets = torch.tensor([2, third, third, 2 * third, rows - 3], dtype=torch.int32, device="cuda")
    clean, grads = check(tw, A, B, offsets, kn), check_gradient(tw, A, dC, offsets, E, kn)
    dirty, d_dirty, b_dirty = A.clone(), dC.clone(), B.clone()
    for t in (dirty, d_dirty):
        t[:2], t[rows - 3:], t[third + 1] = math.nan, math.inf, math.nan    # rows of none, and one of expert 2
    b_dirty[1] = math.nan                                                   # an expert without rows
    got = check(tw, dirty, b_dirty, offsets, kn)
    same = [i for i in range(2, rows - 3) if i != third + 1]
    assert torch.equal(got[same], clean[same]) and bool(got[third + 1].isnan().all())
    got = tw.expert_gemm_backward(dirty, d_dirty, offsets, int(kn))
    assert torch.equal(got[0], grads[0]) and torch.equal(got[3], grads[3]) and bool(got[2].isnan().all()) and not bool(got[1].any())


@pytest.mark.parametrize("wrong", [[-5, 10, 4, 500, 20], [20, 10, 5, 2, 0], [1 << 30] * 5, [-(1 << 31)] * 5, [0, 60, 0, 60, 60],
                                   [(1 << 31) - 1, 0, -(1 << 31), 7, 60]])
def test_wrong_offsets_are_read_as_ascending_ones(tw, wrong):
    g = torch.Generator().manual_seed(6)
    for rows, N, K in ((60, 72, 64), (600, 264, 128)):
        print(wrong, rows, flush=True)
        A, B, dC = normal(g, rows, K), weights(g, 4, N, K, False), normal(g, rows, N)
        offsets = torch.tensor(wrong, dtype=torch.int32, device="cuda")
        check(tw, A, B, offsets, False)
        check_gradient(tw, A, dC, offsets, 4, False)


def test_the_gradient_of_the_rows(tw):
    """dA = dC B^T: the same product with the other layout; against the sum's differences, which are exact for what is linear."""
    g = torch.Generator().manual_seed(7)
    rows, E, N, K = 24, 3, 16, 24
    for kn in (False, True):
        A, B, dC = exact_inputs(g, rows, K), exact_inputs(g, *((E, K, N) if kn else (E, N, K))), exact_inputs(g, rows, N)
        offsets = torch.tensor([0, 9, 9, rows], dtype=torch.int32, device="cuda")
        dA = tw.expert_gemm(dC, B, offsets, int(not kn))
        dB = tw.expert_gemm_backward(A, dC, offsets, int(kn))

        def loss(a, b):
            return sum((a[lo:hi] @ (b[e] if kn else b[e].t()) * dC[lo:hi].double().cpu()).sum() for e, lo, hi in L.rows_of(offsets, rows))

        a, b = A.double().cpu(), B.double().cpu()
        for i in range(rows):
            for j in range(0, K, 7):
                up, down = a.clone(), a.clone()
                up[i, j] += 1
                down[i, j] -= 1
                want = float(loss(up, b) - loss(down, b)) / 2
                assert abs(float(dA[i, j]) - want) <= L.BF16 * abs(want), (i, j)
        for e in range(E):
            for i in range(0, dB.shape[1], 5):
                for j in range(0, dB.shape[2], 5):
                    up, down = b.clone(), b.clone()
                    up[e, i, j] += 1
                    down[e, i, j] -= 1
                    want = float(loss(a, up) - loss(a, down)) / 2
                    assert abs(float(dB[e, i, j]) - want) <= L.BF16 * abs(want), (e, i, j)


def test_captured_calls_serve_other_offsets(tw):
    """Replays with the program's own work between them, and other offsets each time, of products and gradients in one graph."""
    g = torch.Generator().manual_seed(8)
    for rows, E, N, K in ((20, 8, 128, 256), (500, 4, 136, 512), (3000, 4, 520, 264)):
        A, B, dC = normal(g, rows, K), weights(g, E, N, K, False), normal(g, rows, N)
        offsets = counted(g, rows, E)
        C, dB = torch.zeros(rows, N, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(B)
        tw.expert_gemm(A, B, offsets, C=C)
        tw.expert_gemm_backward(A, dC, offsets, dB=dB)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            tw.expert_gemm(A, B, offsets, C=C)
            tw.expert_gemm_backward(A, dC, offsets, dB=dB)
        for i in range(4):
            other = counted(g, rows, E, ahead=i)
            offsets.copy_(other)
            C.fill_(math.nan)
            dB.fill_(math.nan)
            graph.replay()
            torch.cuda.synchronize()
            want = torch.full_like(C, math.nan)
            tw.expert_gemm(A, B, other, C=want)
            assert torch.equal(C.nan_to_num(9.0), want.nan_to_num(9.0)), i
            assert torch.equal(dB, tw.expert_gemm_backward(A, dC, other)), i
            R.assert_close(C, *L.product(A, B, other, False), "replay")


def test_two_streams_and_two_calls_at_once(tw):
    g = torch.Generator().manual_seed(9)
    A, B, offsets = normal(g, 900, 512), weights(g, 6, 264, 512, False), counted(g, 900, 6)
    want = tw.expert_gemm(A, B, offsets)
    dC = normal(g, 900, 264)
    want_dB = tw.expert_gemm_backward(A, dC, offsets)
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for i in range(6):
        s = streams[i % 2]
        C, dB = torch.zeros_like(want), torch.zeros_like(want_dB)
        torch.cuda.synchronize()
        tw.expert_gemm(A, B, offsets, C=C, stream=s)
        tw.expert_gemm_backward(A, dC, offsets, dB=dB, stream=s)
        got.append((C, dB))
    torch.cuda.synchronize()
    for C, dB in got:
        assert torch.equal(C, want) and torch.equal(dB, want_dB)


@pytest.mark.parametrize("kn", [False, True])
def test_weights_beyond_4_gib_and_rows_beyond_4_gib(tw, kn):
    """The last expert's weights, and the last rows, lie further than 32-bit offsets reach."""
    E, N, K = 40, 8192, 8192
    B = torch.zeros(E, N, K, dtype=torch.bfloat16, device="cuda")
    assert (E - 1) * N * K * 2 > 1 << 32
    g = torch.Generator().manual_seed(10)
    B[E - 1] = exact_inputs(g, N, K)
    A = exact_inputs(g, 40, K)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[E] = 40
    want = (A.float() @ (B[E - 1].float() if kn else B[E - 1].float().t())).bfloat16()
    assert torch.equal(tw.expert_gemm(A, B, offsets, int(kn)), want)
    dB = tw.expert_gemm_backward(A, A, offsets, int(kn))
    assert torch.equal(dB[E - 1], (A.float().t() @ A.float()).bfloat16()) and not bool(dB[:E - 1].any())
    del B, dB
    rows, W = 600000, 4096
    assert (rows - 40) * W * 2 > 1 << 32
    A, B = torch.zeros(rows, W, dtype=torch.bfloat16, device="cuda"), exact_inputs(g, 2, W, W)
    A[rows - 40:] = exact_inputs(g, 40, W)
    offsets = torch.tensor([rows - 40, rows - 39, rows], dtype=torch.int32, device="cuda")
    C = tw.expert_gemm(A, B, offsets, int(kn), C=torch.zeros_like(A))
    for e, lo, hi in L.rows_of(offsets, rows):
        assert torch.equal(C[lo:hi], (A[lo:hi].float() @ (B[e].float() if kn else B[e].float().t())).bfloat16())
    assert not bool(C[:rows - 40].any())
    dB = tw.expert_gemm_backward(A, A, offsets)
    assert torch.equal(dB[1], (A[rows - 39:].float().t() @ A[rows - 39:].float()).bfloat16())
