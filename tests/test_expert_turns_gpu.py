"""The experts' products and the gradient of their weights where a workgroup takes several large tiles, one after the other, of experts of
different lengths, with more experts than the lanes of a wave; and which tiles the tests' sizes take."""
import math

import pytest
import torch

import layer_reference as L
import operator_reference as R
from test_expert_tiles_gpu import GRADIENTS, PRODUCTS, whole

CUS = 256
ALL_TILES = {(16, 32), (16, 64), (32, 128), (128, 128), (192, 128), (256, 256)}

# lengths, N, K. Depths (K of a product, rows of a gradient) are several steps of 64 and no multiples of it.
LARGE_PRODUCTS = [([3000, 1, 0, 2500, 700, 64, 257], 3112, 840), ([5001, 1, 0, 4097], 4104, 712),
                  ([0, 1, 255, 256, 257, 600, 900, 1029, 1500, 130] * 7, 1032, 328)]
LARGE_GRADIENTS = [([700, 1, 1500], 3592, 4104), ([0, 1, 63, 64, 65, 130, 777, 1000, 500, 1500] * 7, 520, 776)]
AHEAD, BEHIND = 2, 4    # rows of no expert


def rows_of(lengths):
    return AHEAD + sum(lengths) + BEHIND


def test_every_tile_is_met():
    from paper_2505_11329_amd import expert_gemm_plan
    for kn in (0, 1):
        met = {(f.tile_rows, f.tile_cols) for rows, E, N, K in PRODUCTS for f in (expert_gemm_plan(rows, N, K, E, kn, False, CUS),)}
        assert met == ALL_TILES, (kn, ALL_TILES - met)
        met = {f.tile_rows for lengths, N, K in GRADIENTS for f in (expert_gemm_plan(sum(lengths) + 6, N, K, len(lengths), kn, True, CUS),)}
        assert met == {128, 256}, kn
        for lengths, N, K in LARGE_PRODUCTS:
            f = expert_gemm_plan(rows_of(lengths), N, K, len(lengths), kn, False, CUS)
            there = sum(-(-n // 256) for n in lengths) * -(-N // 256)
            assert (f.tile_rows, f.tile_cols) == (256, 256) and f.workgroups == CUS and there > CUS * 5 // 4, (lengths, kn)
        for lengths, N, K in LARGE_GRADIENTS:
            f = expert_gemm_plan(rows_of(lengths), N, K, len(lengths), kn, True, CUS)
            assert f.tile_rows == 256 and f.workgroups == CUS and f.tiles > 2 * CUS, (lengths, kn)


@pytest.mark.gpu
@pytest.mark.parametrize("kn", [False, True])
@pytest.mark.parametrize("lengths,N,K", LARGE_PRODUCTS)
def test_products_of_several_large_tiles_to_a_workgroup(tw, lengths, N, K, kn):
    """Equal to the last bit on whole numbers; NaN in rows of none, in the weights of an expert without rows and in one row stays there."""
    g = torch.Generator().manual_seed(N)
    E, rows = len(lengths), rows_of(lengths)
    A, B, offsets = whole(g, rows, K), whole(g, *((E, K, N) if kn else (E, N, K))), R.offsets(lengths, AHEAD).cuda()
    want = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    for e, lo, hi in L.rows_of(offsets, rows):
        want[lo:hi] = (A[lo:hi].float() @ (B[e].float() if kn else B[e].float().t())).bfloat16()
    A[:AHEAD], A[rows - BEHIND:], B[lengths.index(0)] = math.nan, math.inf, math.nan
    for _ in range(2):
        assert torch.equal(tw.expert_gemm(A, B, offsets, int(kn), C=torch.full_like(want, 7.0)), want)
    middle = rows // 2
    A[middle] = math.nan
    got = tw.expert_gemm(A, B, offsets, int(kn), C=torch.full_like(want, 7.0))
    keep = torch.arange(rows, device="cuda") != middle
    assert torch.equal(got[keep], want[keep]) and bool(got[middle].isnan().all())


@pytest.mark.gpu
@pytest.mark.parametrize("kn", [False, True])
@pytest.mark.parametrize("lengths,N,K", LARGE_GRADIENTS)
def test_gradients_of_several_large_tiles_to_a_workgroup(tw, lengths, N, K, kn):
    g = torch.Generator().manual_seed(N)
    E, rows = len(lengths), rows_of(lengths)
    A, dC, offsets = whole(g, rows, K), whole(g, rows, N), R.offsets(lengths, AHEAD).cuda()
    want = torch.zeros((E, K, N) if kn else (E, N, K), dtype=torch.bfloat16, device="cuda")
    for e, lo, hi in L.rows_of(offsets, rows):
        x, d = A[lo:hi].float(), dC[lo:hi].float()
        want[e] = (x.t() @ d if kn else d.t() @ x).bfloat16()
    for t in (A, dC):
        t[:AHEAD], t[rows - BEHIND:] = math.nan, math.inf
    for _ in range(2):
        assert torch.equal(tw.expert_gemm_backward(A, dC, offsets, int(kn), dB=torch.full_like(want, math.nan)), want)
