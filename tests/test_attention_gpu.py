"""tw_attention against the plain 64-bit form: lengths, heads, head sizes, masks, strides, and what it leaves alone."""
import ctypes
import math

import pytest
import torch

import operator_reference as R

pytestmark = pytest.mark.gpu


def inputs(q_lens, k_lens, heads, kv_heads, dim, seed=0, tail=0, spread=1.0):
    """bf16 normals on the GPU; `tail` rows more than the sequences have, before and behind them."""
    g = torch.Generator().manual_seed(seed)
    T, Tk = sum(q_lens) + 2 * tail, sum(k_lens) + 2 * tail

    def normal(*shape):
        return (torch.randn(*shape, generator=g) * spread).bfloat16().cuda()

    return (normal(T, heads, dim), normal(Tk, kv_heads, dim), normal(Tk, kv_heads, dim), R.offsets(q_lens, tail).cuda(),
            R.offsets(k_lens, tail).cuda())


def check(tw, q, k, v, qo, ko, causal=True, scale=None, what="", **more):
    out, lse = tw.attention(q, k, v, qo, ko, causal=causal, scale=scale, **more)
    torch.cuda.synchronize()
    c = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    want, want_lse, tol, tol_lse = R.attention(q, k, v, qo, ko, causal, c)
    a, b = int(qo[0]), int(qo[-1])
    R.assert_close(out[a:b], want[a:b], tol[a:b], what + " out")
    R.assert_close(lse[a:b], want_lse[a:b], tol_lse[a:b], what + " lse")
    return out, lse


LENGTHS = [
    ([1], [1]), ([1], [0]), ([2], [1]), ([63], [63]), ([65], [64]), ([5, 0, 1, 130], [5, 7, 33, 130]),
    ([1, 1, 1, 1, 1], [1, 31, 32, 129, 700]), ([257], [257]), ([40, 300], [900, 301]), ([7, 9], [3, 0]), ([0, 0, 3], [4, 0, 3]),
    ([2, 0, 0, 1, 0], [50, 3, 0, 700, 9]), ([1, 1, 0, 0], [600, 40, 7, 0]), ([0, 1], [3, 2]),
]
HEADS = [(1, 1, 64), (4, 2, 128), (8, 1, 128), (6, 2, 72), (3, 3, 8), (32, 1, 64), (5, 1, 96)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
def test_lengths_and_heads(tw, heads, kv_heads, dim, causal):
    for n, (q_lens, k_lens) in enumerate(LENGTHS):
        print(heads, kv_heads, dim, causal, q_lens, k_lens, flush=True)
        args = inputs(q_lens, k_lens, heads, kv_heads, dim, seed=n)
        check(tw, *args, causal=causal, what="%s %s" % (q_lens, k_lens))


@pytest.mark.parametrize("q_lens,k_lens,heads,kv_heads,dim", [
    ([1, 1, 1], [5000, 3, 1300], 8, 1, 128),        # few rows, long keys: the keys are cut into chunks
    ([1], [20011], 4, 4, 64),
    ([100], [4100], 16, 2, 128),                    # a chunk of a prompt, cut too
    ([2, 3, 1, 4], [600, 2049, 1, 1024], 8, 2, 80),
    ([1000, 40], [1000, 2040], 8, 2, 128),          # a prompt and a chunk
    ([300] * 4, [300] * 4, 16, 16, 64),
    ([2200, 1900], [2200, 2400], 32, 8, 128),       # tiles enough for eight waves each
])
def test_long_keys(tw, q_lens, k_lens, heads, kv_heads, dim):
    for causal in (True, False):
        print(q_lens, k_lens, causal, flush=True)
        check(tw, *inputs(q_lens, k_lens, heads, kv_heads, dim, seed=7), causal=causal, what=str(k_lens))


def test_more_keys_than_the_last_level_cache_holds(tw):
    """Single tokens whose keys and values are streamed past the caches."""
    q, k, v, qo, ko = inputs([1, 0, 1], [23000, 5, 18001], 16, 16, 128, seed=1)
    assert k.numel() * 4 > 256 << 20
    check(tw, q, k, v, qo, ko, what="streamed")


@pytest.mark.parametrize("most", [0, 1, 2, 40])
def test_more_sequences_than_lanes(tw, most):
    """Of 150 sequences, single tokens with empty ones behind them, or up to `most` rows in any order."""
    g = torch.Generator().manual_seed(most)
    q_lens = [1] * 130 + [0] * 20 if most == 0 else torch.randint(0, most + 1, (150,), generator=g).tolist()
    k_lens = [n + int(x) for n, x in zip(q_lens, torch.randint(0, 200, (150,), generator=g))]
    check(tw, *inputs(q_lens, k_lens, 4, 2, 64, seed=most), what=str(most))
    check(tw, *inputs(q_lens, k_lens, 24, 1, 64, seed=most), causal=False, what=str(most))


@pytest.mark.parametrize("q_lens,k_lens,heads,kv_heads,dim,tail", [
    ([1] * 20, [300] * 20, 8, 4, 128, 40),                              # rows enough for more tiles than there are sequences
    ([1, 1, 0, 0, 0, 1, 0, 0], [700, 9, 4, 0, 1, 2100, 1, 1], 40, 1, 64, 0),   # a row's heads are more than a tile
    ([60] + [1] * 39, [60] + [90] * 39, 8, 4, 64, 0),                   # one sequence of many tiles
    ([4, 3, 5, 4], [900, 2300, 5, 1700], 16, 4, 128, 0),                # some rows each, keys in parts
    ([9, 0, 2], [4000, 3, 300], 8, 2, 128, 2),
])
def test_few_rows(tw, q_lens, k_lens, heads, kv_heads, dim, tail):
    for causal in (True, False):
        q, k, v, qo, ko = inputs(q_lens, k_lens, heads, kv_heads, dim, seed=9, tail=tail)
        assert tw.attention_plan(len(q_lens), q.shape[0], k.shape[0], heads, kv_heads, dim).key_waves == 4
        check(tw, q, k, v, qo, ko, causal=causal, what=str(q_lens))


def test_forms_of_the_launch(tw):
    """Each kernel and rule is reached by the sizes of these tests."""
    forms = {(f.tile_rows, f.key_waves, f.chunks > 1): sizes for sizes in (
        (1, 1, 1, 8, 1, 128), (1, 1, 20011, 4, 4, 64), (1, 1, 1, 32, 1, 64), (1, 1, 9000, 32, 1, 64), (1, 63, 63, 1, 1, 64),
        (1, 100, 4100, 16, 2, 64), (2, 4100, 4600, 32, 8, 128), (1, 100, 4100, 16, 2, 128), (4, 100, 4000, 4, 2, 128))
        for f in (tw.attention_plan(*sizes),)}
    assert set(forms) == {(16, 4, False), (16, 4, True), (32, 4, False), (32, 4, True), (128, 1, False), (128, 1, True), (256, 1, False),
                          (256, 1, True)}, forms


@pytest.mark.parametrize("q_lens,k_lens", [([1, 1], [40, 2000]), ([150, 3], [150, 90])])
def test_scores_far_apart_and_scale(tw, q_lens, k_lens):
    # scores of some hundreds: one key has all the weight, and the running maximum changes from tile to tile
    check(tw, *inputs(q_lens, k_lens, 4, 2, 128, seed=3, spread=6.0), what="far apart")
    check(tw, *inputs(q_lens, k_lens, 4, 2, 64, seed=4), scale=0.02, what="flat")
    # a maximum that grows with every key, and one that comes first
    for order in (1, -1):
        q, k, v, qo, ko = inputs(q_lens, k_lens, 2, 1, 64, seed=5)
        ramp = torch.linspace(-4, 4, k.shape[0], device="cuda")[::1 if order == 1 else -1] if order == 1 else torch.linspace(4, -4, k.shape[0], device="cuda")
        k = ramp[:, None, None].expand_as(k).bfloat16().contiguous()
        check(tw, q.abs(), k, v, qo, ko, what="ramp")


def test_rows_and_memory_outside_the_sequences_are_left_alone(tw):
    for q_lens, k_lens, heads in (([3, 70], [90, 70], 4), ([1, 1], [900, 1500], 4)):
        q, k, v, qo, ko = inputs(q_lens, k_lens, heads, 2, 64, tail=5)
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        for t in (k, v):        # NaN around the sequences' keys
            t[:5], t[-5:] = math.nan, math.nan
        check(tw, q, k, v, qo, ko, out=out, lse=lse, what="tail")
        for t in (out, lse):
            assert bool((t[:5] == 7).all()) and bool((t[-5:] == 7).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("q_lens,k_lens,heads,dim", [([130, 20], [130, 90], 2, 128), ([2, 2, 4], [33, 900, 64], 8, 64),
                                                    ([4], [3000], 4, 128)])
def test_keys_that_a_row_does_not_see_have_no_part_in_it(tw, bad, q_lens, k_lens, heads, dim):
    """Inf and NaN at the last key of each sequence: seen by its last row only."""
    q, k, v, qo, ko = inputs(q_lens, k_lens, heads, 2, dim, seed=11)
    ends = (ko[1:] - 1).long()
    rows = (qo[1:] - 1).long()
    clean, clean_lse = tw.attention(q, k, v, qo, ko)
    v2, k2 = v.clone(), k.clone()
    v2[ends, :, 1::2] = bad
    out, lse = check(tw, q, k, v2, qo, ko, what="v")
    others = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    others[rows] = False
    assert torch.equal(out[others], clean[others]) and torch.equal(lse, clean_lse)
    assert not bool(torch.isfinite(out[rows][:, :, 1::2]).any())
    k2[ends] = bad
    out, lse = tw.attention(q, k2, v, qo, ko)
    assert torch.equal(out[others], clean[others]) and torch.equal(lse[others], clean_lse[others])


def test_nan_in_a_query_row_stays_there(tw):
    for q_lens, k_lens in (([70], [70]), ([1, 1], [50, 60])):
        q, k, v, qo, ko = inputs(q_lens, k_lens, 4, 2, 64, seed=2)
        clean, _ = tw.attention(q, k, v, qo, ko)
        q2 = q.clone()
        q2[-1, 2] = math.nan
        out, lse = tw.attention(q2, k, v, qo, ko)
        assert bool(torch.isnan(out[-1, 2]).all()) and bool(torch.isnan(lse[-1, 2]))
        out[-1, 2] = clean[-1, 2]
        assert torch.equal(out, clean)


def test_columns_of_one_projection(tw):
    for T, heads, kv_heads, dim in ((77, 6, 2, 64), (300, 8, 4, 128), (1, 4, 1, 24)):
        g = torch.Generator().manual_seed(T)
        qkv = torch.randn(T, heads + 2 * kv_heads, dim, generator=g).bfloat16().cuda()
        q, k, v = qkv.split([heads, kv_heads, kv_heads], dim=1)
        both = torch.zeros(T, 2 * heads, dim, dtype=torch.bfloat16, device="cuda")
        o = R.offsets([T]).cuda()
        check(tw, q, k, v, o, o, out=both[:, heads:], what="packed")
        assert not bool(both[:, :heads].any())


def test_keys_and_values_beyond_32_bit_offsets(tw):
    """Rows 8 MiB apart: the last ones lie more than 4 GiB from the first."""
    T, stride = 600, 1 << 22
    big = torch.empty(T * stride, dtype=torch.bfloat16, device="cuda")
    k, v = big.as_strided((T, 2, 64), (stride, 64, 1)), big.as_strided((T, 2, 64), (stride, 64, 1), 1024)
    q, k0, v0, qo, ko = inputs([3, 200], [350, 250], 4, 2, 64)
    k.copy_(k0)
    v.copy_(v0)
    out, lse = tw.attention(q, k, v, qo, ko)
    want, want_lse = tw.attention(q, k0, v0, qo, ko)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    check(tw, q, k0, v0, qo, ko)


def test_offsets_outside_the_tensors_count_as_their_nearest_row(tw):
    q, k, v, _, _ = inputs([50, 20], [90, 30], 4, 2, 64)
    wild = torch.tensor([-5, 50, 1 << 30], dtype=torch.int32, device="cuda")
    tame = R.offsets([50, 20]).cuda()
    wild_k, tame_k = torch.tensor([-(1 << 31), 90, (1 << 31) - 1], dtype=torch.int32, device="cuda"), R.offsets([90, 30]).cuda()
    for x, y in zip(tw.attention(q, k, v, wild, wild_k), tw.attention(q, k, v, tame, tame_k)):
        assert torch.equal(x, y)


def test_a_batch_split_between_its_sequences_and_inside_one_gives_the_same_bits(tw):
    """The token split: the second half's rows attend to the first half's keys. All three calls have one form."""
    heads, kv_heads, dim = 64, 32, 64
    q, k, v, qo, ko = inputs([1700, 3100], [1900, 3100], heads, kv_heads, dim, seed=9)
    cut, k_cut = 1700 + 1100, 1900 + 1100       # inside the second sequence, with its keys up to there
    forms = [tw.attention_plan(*n, heads, kv_heads, dim) for n in ((2, 4800, 5000), (2, cut, k_cut), (1, 2000, 5000))]
    assert len({(f.tile_rows, f.key_waves, f.chunks) for f in forms}) == 1 and forms[0].chunks == 1
    whole, whole_lse = tw.attention(q, k, v, qo, ko)
    a, a_lse = tw.attention(q[:cut], k[:k_cut], v[:k_cut], R.offsets([1700, 1100]).cuda(), R.offsets([1900, 1100]).cuda())
    b, b_lse = tw.attention(q[cut:], k, v, R.offsets([2000]).cuda(), R.offsets([3100], 1900).cuda())
    assert torch.equal(torch.cat([a, b]), whole) and torch.equal(torch.cat([a_lse, b_lse]), whole_lse)


def test_streams_workspaces_and_graphs(tw):
    """Two streams at once, the workspace from torch or the caller, and a captured call replayed among eager ones."""
    cases = [inputs([1, 1, 1], [3000, 40, 1800], 8, 2, 128, seed=s) for s in (1, 2)] + [inputs([90, 200], [90, 300], 8, 2, 64, seed=3)]
    want = [tw.attention(*c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        got = []
        for c, s in zip(cases, streams):
            out, lse = torch.zeros_like(c[0]), torch.zeros(c[0].shape[:2], device="cuda")
            s.wait_stream(torch.cuda.current_stream())
            got.append(tw.attention(*c, out=out, lse=lse, stream=s))
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
    q, k, v, qo, ko = cases[0]
    need = tw.attention_workspace_bytes(3, q.shape[0], k.shape[0], 8, 2, 128)
    assert need > 0
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    with pytest.raises(tw.TwError) as e:
        tw.attention(*cases[0], workspace=space[:-1])
    assert e.value.status == 2
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        tw.attention(*cases[0], out=out, lse=lse, workspace=space)
    for n in range(4):
        out.fill_(n)
        graph.replay()
        other = tw.attention(*cases[1])
        torch.cuda.synchronize()
        assert torch.equal(out, want[0][0]) and torch.equal(lse, want[0][1]) and torch.equal(other[0], want[1][0])
        q.copy_(cases[1][0] if n % 2 == 0 else inputs([1, 1, 1], [3000, 40, 1800], 8, 2, 128, seed=1)[0])
        want[0] = tw.attention(*cases[0])


@pytest.mark.parametrize("rows,batches", [
    (8, [([1] * 8, [40] * 7 + [2900]), ([1] * 5 + [0] * 3, [9, 3000, 1, 33, 64, 0, 0, 0]), ([0, 4, 0, 1, 3, 0, 0, 0], [5, 900, 0, 1, 700, 0, 2, 0])]),
    (400, [([100] * 4, [100] * 4), ([0, 1, 0, 380], [60, 77, 0, 400]), ([400, 0, 0, 0], [450, 0, 0, 1])]),
])
def test_a_captured_call_replayed_with_other_offsets(tw, rows, batches):
    """The launch depends on the tensors' sizes alone: a graph serves every batch that fits them."""
    n, keys = len(batches[0][0]), max(sum(k) for _, k in batches)
    q, k, v, qo, ko = inputs([rows] + [0] * (n - 1), [keys] + [0] * (n - 1), 8, 2, 64, seed=6)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    space = torch.empty(tw.attention_workspace_bytes(n, rows, keys, 8, 2, 64), dtype=torch.uint8, device="cuda")
    tw.attention(q, k, v, qo, ko, out=out, lse=lse, workspace=space)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tw.attention(q, k, v, qo, ko, out=out, lse=lse, workspace=space)
    for q_lens, k_lens in batches + batches[:1]:
        qo.copy_(R.offsets(q_lens))
        ko.copy_(R.offsets(k_lens))
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        want, want_lse = check(tw, q, k, v, qo, ko, what=str(q_lens))
        end = sum(q_lens)
        assert torch.equal(got[:end], want[:end]) and torch.equal(got_lse[:end], want_lse[:end])
        assert bool((got[end:] == 3).all())


@pytest.mark.parametrize("q_lens,heads,kv_heads,dim,past", [
    ([1, 5], 32, 8, 128, (0, 40)), ([1, 3], 64, 8, 64, (5, 0)), ([1, 1, 3], 64, 8, 128, (900, 12)), ([1, 7], 24, 8, 80, (30, 3000)),
    ([1] * 61 + [5], 8, 1, 64, (7, 90)), ([1] * 40 + [20], 16, 4, 72, (300, 0)), ([1] * 47 + [41], 16, 2, 128, (60, 2000)),
    ([1] * 99 + [60], 16, 2, 64, (33, 500)), ([1] * 256 + [1024], 8, 2, 128, (100, 0)), ([1] * 7 + [2], 23, 1, 128, (2500, 2500)),
])
@pytest.mark.parametrize("spare", [0, 1])
def test_single_tokens_and_a_longer_sequence_behind_them(tw, q_lens, heads, kv_heads, dim, past, spare):
    """The form for few rows, whose tiles are the sequences one by one only where every one of them has a single row."""
    k_lens = [n + past[i == len(q_lens) - 1] for i, n in enumerate(q_lens)]
    q, k, v, qo, ko = inputs(q_lens, k_lens, heads, kv_heads, dim, seed=12, tail=spare)
    sizes = len(q_lens), q.shape[0], k.shape[0], heads, kv_heads, dim
    assert tw.attention_plan(*sizes).key_waves == 4
    for causal in (True, False):
        print(q_lens[:3], len(q_lens), causal, flush=True)
        out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device="cuda")
        space = torch.full((tw.attention_workspace_bytes(*sizes),), 255, dtype=torch.uint8, device="cuda")   # NaN, too
        check(tw, q, k, v, qo, ko, causal=causal, out=out, lse=lse, workspace=space, what="%s %s" % (q_lens[-1], causal))


@pytest.mark.parametrize("group,most", [(4, 70), (8, 700)])
def test_a_captured_call_of_single_tokens_replayed_with_a_longer_sequence_behind_them(tw, group, most):
    n, rows, keys = 40, 78, 40 * most + 100
    q, k, v, qo, ko = inputs([rows] + [0] * (n - 1), [keys] + [0] * (n - 1), group, 1, 64, seed=8)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    space = torch.full((tw.attention_workspace_bytes(n, rows, keys, group, 1, 64),), 255, dtype=torch.uint8, device="cuda")
    assert tw.attention_plan(n, rows, keys, group, 1, 64).key_waves == 4
    tw.attention(q, k, v, qo, ko, out=out, lse=lse, workspace=space)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tw.attention(q, k, v, qo, ko, out=out, lse=lse, workspace=space)
    for q_lens in ([1] * n, [1] * (n - 1) + [39], [1] * 20 + [0] * 20, [1] * (n - 1) + [2], [0] + [1] * (n - 1), [1] * n):
        k_lens = [x + most - 60 + i for i, x in enumerate(q_lens)]
        qo.copy_(R.offsets(q_lens))
        ko.copy_(R.offsets(k_lens))
        out.fill_(math.nan)
        lse.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        end = sum(q_lens)
        want, want_lse, tol, tol_lse = R.attention(q, k, v, qo, ko, True, 0.125)
        R.assert_close(out[:end], want[:end], tol[:end], "out %s" % q_lens)
        R.assert_close(lse[:end], want_lse[:end], tol_lse[:end], "lse %s" % q_lens)
        assert bool(torch.isnan(out[end:]).all()) and bool(torch.isnan(lse[end:]).all())


def test_offsets_outside_the_tensors_in_the_form_for_few_rows(tw):
    """Taken as their nearest rows, these are single tokens and empty sequences around them."""
    for rows, wild, tame in ((2, [-1, 0, 1, 2, 2], [0, 0, 1, 2, 2]), (3, [-9, -4, 1, 2, 3, 1 << 30], [0, 0, 1, 2, 3, 3]),
                             (3, [0, 1, 2, 5, 9], [0, 1, 2, 3, 3])):
        k_lens = [50, 3, 700, 33, 5][:len(wild) - 1]
        q, k, v, _, ko = inputs([rows] + [0] * (len(wild) - 2), k_lens, 8, 2, 64, seed=rows)
        assert tw.attention_plan(len(k_lens), rows, k.shape[0], 8, 2, 64).key_waves == 4
        wild, tame = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (wild, tame))
        want = check(tw, q, k, v, tame, ko, what=str(tame.tolist()))
        got = tw.attention(q, k, v, wild, ko, out=torch.full_like(q, math.nan), lse=torch.full(q.shape[:2], math.nan, device="cuda"))
        for x, y in zip(got, want):
            assert torch.equal(x, y)


# one of each way to read the keys: four and eight waves of 32 rows, whole keys and parts; few rows, whole keys and parts
FORMS = [(200, 320, 2, 1, 64), (200, 320, 4, 4, 128), (2048, 2112, 32, 32, 128), (100, 4096, 16, 2, 128), (100, 4160, 16, 2, 128),
         (100, 4096, 16, 2, 64), (4, 256, 4, 2, 64),
         (4, 256, 8, 1, 128), (3, 2048, 16, 2, 128), (2, 2048, 8, 1, 64)]


@pytest.mark.parametrize("rows,keys,heads,kv_heads,dim", FORMS)
def test_inf_in_values_of_any_weight_whatever_the_rows_around(tw, rows, keys, heads, kv_heads, dim):
    """A key that a row sees, with Inf, -Inf and NaN among its values: Inf where its weight is one in fp32, NaN where it is
    too small for that, and the same whether the rows of the tile see all of the tile's keys (no mask; the number of keys is a
    multiple of every tile) or a part of them (a mask, which hides none from the last row)."""
    assert keys % 64 == 0
    g = torch.Generator().manual_seed(keys)
    q = torch.zeros(rows, heads, dim, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 1
    v = torch.randn(keys, kv_heads, dim, generator=g).bfloat16().cuda()
    at = keys - 6
    v[at, :, 0], v[at, :, 1], v[at, :, 2], v[at, :, 3] = math.inf, -math.inf, math.nan, math.inf
    v[at + 1, :, 3] = -math.inf
    o = [R.offsets([n]).cuda() for n in (rows, keys)]
    for best in (0, at - 9, keys - 1):       # the key with all of the weight
        for gap in (0, 20, 64, 80, 86, 87, 88, 90, 92, 96, 100, 104, 120, 200, 1000):
            k = torch.zeros(keys, kv_heads, dim, dtype=torch.bfloat16, device="cuda")
            k[:, :, 0] = -gap
            k[best, :, 0] = 0
            got = [tw.attention(q, k, v, *o, causal=causal, scale=1.0) for causal in (True, False)]
            last = [(out[-1], lse[-1]) for out, lse in got]
            print(rows, keys, best, gap, last[0][0][0, :4].tolist(), last[1][0][0, :4].tolist(), flush=True)
            for a, b in zip(*last):
                assert torch.equal(torch.nan_to_num(a, 3e38, 2e38, -2e38), torch.nan_to_num(b, 3e38, 2e38, -2e38))
            out, lse = last[0]
            assert bool(torch.isfinite(out[:, 4:]).all()) and bool(torch.isfinite(lse).all())
            assert bool(torch.isnan(out[:, 2:4]).all())
            if gap <= 80:            # e^-80 is a number of fp32, e^-120 is none
                assert bool((out[:, 0] == math.inf).all()) and bool((out[:, 1] == -math.inf).all())
            elif gap >= 120:
                assert bool(torch.isnan(out[:, :2]).all())
            # rows that the mask hides those keys from
            assert bool(torch.isfinite(got[0][0][:max(rows - 6, 0)]).all())


@pytest.mark.parametrize("rows,keys,heads,kv_heads,dim", FORMS + [(1, 1, 2, 2, 64), (70, 1, 2, 1, 128)])
def test_scores_whose_steps_are_large(tw, rows, keys, heads, kv_heads, dim):
    """Scores whose neighbouring numbers in fp32 are far apart: the key with the largest one has all of the weight. Its p is
    rounded to bf16 and so is the result; lse is the score, rounded three times, and a sum of 1."""
    g = torch.Generator().manual_seed(rows)
    q, k = (torch.zeros(n, h, dim, dtype=torch.bfloat16, device="cuda") for n, h in ((rows, heads), (keys, kv_heads)))
    v = torch.randn(keys, kv_heads, dim, generator=g).bfloat16().cuda()
    o = [R.offsets([n]).cuda() for n in (rows, keys)]
    for power in (20, 25, 28, 31, 34, 40, 60, 100, 122):
        for sign, best, others in ((1.3, 1.7, 1.0), (-1.3, 1.0, 1.7)):
            for at in (0, keys - 1):
                print(rows, keys, power, sign, at, flush=True)
                q[:, :, 0], k[:, :, 0] = sign * 2.0 ** (power // 2), others * 2.0 ** (power - power // 2)
                k[at, :, 0] = best * 2.0 ** (power - power // 2)
                out, lse = tw.attention(q, k, v, *o, causal=False, scale=0.3)
                want = v[at].double().repeat_interleave(heads // kv_heads, dim=0).expand(rows, heads, dim)
                R.assert_close(out, want, (2 * R.BF16 + 2.0 ** -15) * want.abs(), "out")
                score = float(torch.tensor(0.3)) * float(q[0, 0, 0].double() * k[at, 0, 0].double())
                want_lse = torch.full((rows, heads), score, dtype=torch.float64, device="cuda")
                R.assert_close(lse, want_lse, 4 * R.F32 * want_lse.abs() + 2.0 ** -20, "lse")


@pytest.mark.parametrize("rows,keys,heads,kv_heads,dim", FORMS)
def test_scores_beyond_fp32(tw, rows, keys, heads, kv_heads, dim):
    """Scores that overflow give NaN, as Inf - Inf does; a row all of whose scores are -Inf counts as one that sees no key."""
    q, k = (torch.zeros(n, h, dim, dtype=torch.bfloat16, device="cuda") for n, h in ((rows, heads), (keys, kv_heads)))
    v = torch.ones_like(k)
    o = [R.offsets([n]).cuda() for n in (rows, keys)]
    q[:, :, 0] = 2.0 ** 63
    k[0, :, 0] = 2.0 ** 63      # 2^126 is a number of fp32, four times that is none
    minus_inf = torch.full_like(k, -math.inf)
    for causal in (True, False):
        out, lse = tw.attention(q, k, v, *o, causal=causal, scale=1.0)
        assert bool((out == 1).all()) and bool(torch.isfinite(lse).all())
        out, lse = tw.attention(q, k, v, *o, causal=causal, scale=4.0)
        assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())
        out, lse = tw.attention(torch.ones_like(q), minus_inf, v, *o, causal=causal)
        assert not bool(out.any()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("rows,keys,heads,kv_heads,dim", FORMS)
def test_no_lse_and_results_between_other_columns(tw, rows, keys, heads, kv_heads, dim):
    """The C call without lse, results in rows that are longer than theirs, in every form."""
    q, k, v, qo, ko = inputs([rows], [keys], heads, kv_heads, dim, seed=keys, tail=1)
    wide = torch.full((rows + 2, heads + 2, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, 1:heads + 1]
    want, _ = tw.attention(q, k, v, qo, ko)
    a = tw.AttentionArgs(q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), out=out.data_ptr(), lse=None, q_offsets=qo.data_ptr(),
                         k_offsets=ko.data_ptr(), n_seqs=1, q_rows=rows + 2, k_rows=keys + 2, q_stride=heads * dim, k_stride=kv_heads * dim,
                         v_stride=kv_heads * dim, out_stride=(heads + 2) * dim, q_heads=heads, kv_heads=kv_heads, head_dim=dim,
                         scale=1.0 / math.sqrt(dim), causal=1)
    need = tw.lib().tw_attention_workspace_bytes(ctypes.byref(a))
    space = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert tw.lib().tw_attention(ctypes.byref(a), ctypes.c_void_p(space.data_ptr()), need, stream) == 0
    assert torch.equal(out[1:-1], want[1:-1])
    out[1:-1] = 7.0
    assert bool((wide == 7).all())
