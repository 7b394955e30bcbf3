"""The experts' products and the gradient of their weights at sizes that between them take every tile of the launch's choice, edges in all three
dimensions, experts of no row, of one and of most."""
import math

import pytest
import torch

import layer_reference as L
import operator_reference as R

pytestmark = pytest.mark.gpu


def whole(g, *shape):
    """Small whole numbers: every sum of them is exact in fp32, whatever its order."""
    return torch.randint(-3, 4, shape, generator=g).to(torch.bfloat16).cuda()


def spread_offsets(g, rows, E, ahead, behind):
    cuts = sorted(torch.randint(ahead, rows - behind + 1, (E - 1,), generator=g).tolist())
    return torch.tensor([ahead] + cuts + [rows - behind], dtype=torch.int32).cuda()


# rows, experts, N, K: tiles of 16 x 32, 16 x 64, 32 x 128, 128 x 128, 192 x 128 and 256 x 256 for one layout of the weights or both
PRODUCTS = [(14, 2, 24, 376), (4238, 5, 8, 352), (2336, 3, 40, 376), (4327, 5, 80, 328), (191, 9, 2928, 432), (2514, 9, 3112, 336), (18, 9, 2344, 360), (41, 9, 976, 392), (18, 9, 2144, 368), (96, 8, 3592, 840), (5323, 5, 112, 328),
            (5644, 5, 296, 328), (448, 9, 2992, 328), (768, 9, 2880, 344), (3163, 9, 2952, 336), (5301, 9, 1424, 336), (2600, 3, 1288, 1096)]


@pytest.mark.parametrize("kn", [False, True])
@pytest.mark.parametrize("rows,E,N,K", PRODUCTS)
def test_products_in_every_tile(tw, rows, E, N, K, kn):
    """Equal to the last bit on whole numbers; NaN in rows of no expert and in a row of another one stays there."""
    g = torch.Generator().manual_seed(rows + N)
    A, B = whole(g, rows, K), whole(g, *((E, K, N) if kn else (E, N, K)))
    for ahead, behind in ((0, 0), (1, min(5, rows // 4))):
        offsets = spread_offsets(g, rows, E, ahead, behind)
        C = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
        want = C.clone()
        for e, lo, hi in L.rows_of(offsets, rows):
            want[lo:hi] = (A[lo:hi].float() @ (B[e].float() if kn else B[e].float().t())).bfloat16()
        assert torch.equal(tw.expert_gemm(A, B, offsets, int(kn), C=C), want), (ahead, behind)
        dirty, middle = A.clone(), rows // 2
        dirty[:ahead], dirty[rows - behind:], dirty[middle] = math.nan, math.inf, math.nan
        got = tw.expert_gemm(dirty, B, offsets, int(kn), C=torch.full_like(C, 7.0))
        keep = torch.arange(rows, device="cuda") != middle
        assert torch.equal(got[keep], want[keep]) and bool(got[middle].isnan().all()), (ahead, behind)


# rows of each expert, N, K: large tiles where experts have 400 rows on average and there are tiles for more than half of the compute units; small ones
GRADIENTS = [([900, 1, 640], 1800, 2056), ([0, 1300], 2312, 2568), ([449], 3080, 3000), ([1025, 0, 7, 1666], 1288, 2184), ([64, 63, 65, 33, 32, 31, 0, 1], 520, 392),
             ([399, 2, 96], 136, 1032), ([4100], 264, 520), ([5, 300, 128, 97, 0, 1] * 12, 200, 776)]


@pytest.mark.parametrize("kn", [False, True])
@pytest.mark.parametrize("lengths,N,K", GRADIENTS)
def test_weight_gradients_in_both_tiles(tw, lengths, N, K, kn):
    g = torch.Generator().manual_seed(len(lengths) + N)
    E, rows = len(lengths), sum(lengths) + 6
    A, dC, offsets = whole(g, rows, K), whole(g, rows, N), R.offsets(lengths, 2).cuda()
    want = torch.zeros((E, K, N) if kn else (E, N, K), dtype=torch.bfloat16, device="cuda")
    for e, lo, hi in L.rows_of(offsets, rows):
        x, d = A[lo:hi].float(), dC[lo:hi].float()
        want[e] = (x.t() @ d if kn else d.t() @ x).bfloat16()
    for t in (A, dC):
        t[:2], t[rows - 4:] = math.nan, math.inf          # rows of none
    for _ in range(2):
        assert torch.equal(tw.expert_gemm_backward(A, dC, offsets, int(kn), dB=torch.full_like(want, math.nan)), want)
    normal_A, normal_dC = (torch.randn(rows, W, generator=g).bfloat16().cuda() for W in (K, N))
    R.assert_close(tw.expert_gemm_backward(normal_A, normal_dC, offsets, int(kn)), *L.weight_gradient(normal_A, normal_dC, offsets, E, kn), "dB")


def test_more_rows_than_small_tiles_are_launched_for(tw):
    """2^26 and some rows of few columns, for which a workgroup to a tile would be too many."""
    g = torch.Generator().manual_seed(12)
    rows = (1 << 26) + 77
    A = whole(g, 4096, 8).repeat((rows + 4095) // 4096, 1)[:rows]
    B, offsets = whole(g, 3, 8, 8), torch.tensor([5, 20_000_001, 20_000_001, rows - 3], dtype=torch.int32).cuda()
    for kn in (False, True):
        C = tw.expert_gemm(A, B, offsets, int(kn), C=torch.full((rows, 8), 7.0, dtype=torch.bfloat16, device="cuda"))
        want = torch.full_like(C, 7.0)
        for e, lo, hi in L.rows_of(offsets, rows):
            want[lo:hi] = (A[lo:hi].float() @ (B[e].float() if kn else B[e].float().t())).bfloat16()
        assert torch.equal(C, want), kn
