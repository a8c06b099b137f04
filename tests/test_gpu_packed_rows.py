"""Rows in 4 bits: packing, looking up, scoring, against the definition in 64 bits.

Tolerances.  Packing: the scale is one quotient in fp32, rounded to its type; q is what fp32 arithmetic says, exactly.  A looked-up
element is two products in fp32 (2^-24 each) and the output's rounding.  A score's group sum has at most 128 terms, exact products
added in fp32 (taken as up to 2^-23 of the running size each, the tensor cores' alignment not being specified),
then one product and one addition per group, the three parts of an fp32 vector and the shares of up to 8 warps.
"""
import itertools

import pytest
import torch

from paper_2209_07663_b200 import binding as mb
from tests.test_gpu_token_rows import BF16, F16, F32, SUBNORMAL, TYPES, randn, some_tokens

pytestmark = pytest.mark.gpu


def packed(rows, cols, group, scales=F16, seed=0, extra=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(0, 256, (rows, (cols + 31) // 32 * 16 + 16 * extra), dtype=torch.uint8, device="cuda", generator=g)
    s = (torch.rand((rows, -(-cols // group) + extra), device="cuda", generator=g) + 0.1) * 0.01
    return q, s.to(scales)


def values(q, scales, group, cols):
    c = torch.arange(cols, device="cuda")
    return ((q[:, c // 2] >> (4 * (c % 2)).to(torch.uint8)) % 16).double() - 8.0, scales[:, c // group].double()


def check_scores(got, q, scales, group, x):
    v, s = values(q, scales, group, x.shape[1])
    want = x.double() @ (v * s).T
    size = x.double().abs() @ (v * s).abs().T
    groups = -(-x.shape[1] // group)
    tol = size * (min(group, x.shape[1]) + groups + 16) * 2.0 ** -23 + want.abs() * (torch.finfo(got.dtype).eps / 2) + SUBNORMAL[got.dtype] / 2
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), f"worst {float((err - tol).max())} of {float(want.abs().max())}"


# ---- packing ----

@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("cols", [1, 2, 31, 32, 33, 100, 128, 200, 515, 1024])
def test_packing(cols, group):
    for k, (w, s) in enumerate(itertools.product(TYPES, TYPES)):
        rows = randn(67, cols, dtype=w, seed=k, scale=0.3)
        rows[5] = 0.0
        padded, groups = (cols + 31) // 32 * 16, -(-cols // group)
        q = torch.full((67, padded + 16), 77, dtype=torch.uint8, device="cuda")
        scales = torch.full((67, groups + 1), 9.0, dtype=s, device="cuda")
        mb.mono_pack_rows(rows, q, scales, group)
        assert bool((q[:, padded:] == 77).all()) and bool((scales[:, groups:] == 9).all())
        full = torch.zeros((67, groups * group), device="cuda")
        full[:, :cols] = rows.float()
        full = full.view(67, groups, group)
        want = (full.abs().amax(2) / torch.tensor(7.0, device="cuda")).to(s)
        assert torch.equal(scales[:, :groups], want)
        by = want.float()[:, :, None]
        quot = torch.where(by > 0, full / torch.where(by > 0, by, 1.0), 0.0)
        want_q = (torch.round(quot).clamp(-7, 7) + 8).view(67, -1).to(torch.uint8)
        halves = torch.full((67, max(groups * group, padded * 2)), 8, dtype=torch.uint8, device="cuda")
        halves[:, :groups * group] = want_q
        halves = halves[:, :padded * 2]
        assert torch.equal(q[:, :padded], halves[:, 0::2] | halves[:, 1::2] << 4)


@pytest.mark.parametrize("scales", TYPES)
def test_packing_rounds_the_quotient_and_not_something_near_it(scales):
    # quotients around every half between -8 and 8: the numbers next to half a scale on both sides
    for top in (7.0, 1.0, 0.1, 3e-5, 1e-38, 1e-44, 5e37):
        rows = torch.zeros((64, 128), device="cuda")
        rows[:, 0] = top
        scale = (rows[:, :1] / torch.tensor(7.0, device="cuda")).to(scales).float()
        halves = (torch.arange(-8, 8, device="cuda") + 0.5).repeat_interleave(4)[None, :] * scale
        near = halves.clone()
        for k in range(64):
            x = near[k].view(torch.int32) + (k % 9 - 4)     # up to four numbers further on
            rows[k, 32:96] = x.view(torch.float32)
        rows = torch.where(rows.abs() <= top, rows, 0.0)
        rows[:, 0] = top
        q, s = torch.empty((64, 64), dtype=torch.uint8, device="cuda"), torch.empty((64, 1), dtype=scales, device="cuda")
        mb.mono_pack_rows(rows, q, s, 128)
        by = s.float()
        usable = (by > 0) & torch.isfinite(by)
        got = torch.stack((q & 15, q >> 4), -1).flatten(1)
        assert torch.equal(got, (torch.where(usable, torch.round(rows / torch.where(usable, by, 1.0)).clamp(-7, 7), 0.0) + 8).to(torch.uint8)), top


def test_packing_what_is_not_finite_or_too_large_or_too_small():
    rows = randn(6, 64)
    rows[0, 3], rows[1, 40], rows[2, 1] = float("nan"), float("inf"), float("-inf")
    rows[3] = 1e6                       # beyond an fp16 scale
    rows[4] = 1e-9                      # below the smallest fp16
    q, scales = torch.empty((6, 32), dtype=torch.uint8, device="cuda"), torch.empty((6, 2), dtype=F16, device="cuda")
    mb.mono_pack_rows(rows, q, scales, 32)
    out = torch.empty((6, 64), device="cuda")
    mb.mono_packed_token_rows(q, scales, 32, torch.arange(6, device="cuda"), out)
    bad = torch.isnan(out).view(6, 2, 32)
    assert bad.all(2).tolist() == [[True, False], [False, True], [True, False], [True, True], [False, False], [False, False]]
    assert bad.any(2).tolist() == bad.all(2).tolist()
    assert bool((out[4] == 0).all()) and bool((q[4] == 0x88).all())
    assert bool(((out[5] - rows[5]).abs().view(2, 32) <= scales[5].float()[:, None] * (0.5 + 2.0 ** -8)).all())


# ---- lookup ----

@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("cols", [1, 2, 7, 8, 31, 64, 100, 257, 515, 1024])
def test_packed_rows(cols, group):
    for k, (s, o) in enumerate(itertools.product(TYPES, TYPES)):
        n = (1, 5, 300)[k % 3]
        q, scales = packed(200, cols, group, s, seed=k, extra=k % 2)
        tokens = some_tokens(n, 200, (torch.int64, torch.int32)[k % 2], seed=k)
        out = torch.full((n + 2, cols), 7.0, dtype=o, device="cuda")
        mb.mono_packed_token_rows(q, scales, group, tokens, out[:n], scale=1.3, padding=9)
        t = tokens.long()
        there = (t >= 0) & (t < 200) & (t != 9)
        want = torch.zeros((n, cols), dtype=torch.float64, device="cuda")
        v, f = values(q, scales, group, cols)
        want[there] = (v * f)[t[there]] * float(torch.tensor(1.3))
        tol = want.abs() * (torch.finfo(o).eps / 2 + 2.0 ** -22) + SUBNORMAL[o] / 2
        assert bool(((out[:n].double() - want).abs() <= tol).all())
        assert bool((out[n:] == 7).all())
        assert not bool(torch.signbit(out[:n][~there]).any())


def test_packed_rows_with_strides_and_behind_the_32nd_bit():
    rows, cols = (1 << 32) // 2048 + 100, 4096
    q = torch.zeros((rows, 2048), dtype=torch.uint8, device="cuda")
    scales = torch.ones((rows, 32), dtype=F16, device="cuda")
    at = torch.tensor([rows - 1, 0, (1 << 31) // 2048, (1 << 32) // 2048 + 1], device="cuda")
    q[at] = torch.randint(0, 256, (4, 2048), dtype=torch.uint8, device="cuda")
    store = torch.full((4, cols + 3), 5.0, device="cuda")
    mb.mono_packed_token_rows(q, scales, 128, at, store[:, 1:cols + 1])
    v, _ = values(q[at], scales[at], 128, cols)
    assert torch.equal(store[:, 1:cols + 1].double(), v)
    assert bool((store[:, 0] == 5).all()) and bool((store[:, cols + 1:] == 5).all())


# ---- scores ----

@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("cols", [1, 2, 31, 32, 33, 64, 100, 128, 130, 257, 515, 1000, 2048])
@pytest.mark.parametrize("m", [1, 2, 3, 8, 9, 16])
def test_scores(m, cols, group):
    for k, (s, t) in enumerate(itertools.product(TYPES, TYPES)):
        rows = (1, 15, 16, 17, 333, 2000, 130, 64, 128)[k]
        q, scales = packed(rows, cols, group, s, seed=k, extra=k % 2)
        x = randn(m, cols, dtype=t, seed=k)
        store = torch.full((m + 1, rows + 3), 7.0, dtype=TYPES[(k + m) % 3], device="cuda")
        mb.mono_packed_scores(q, scales, group, x, store[:m, :rows])
        check_scores(store[:m, :rows], q, scales, group, x)
        assert bool((store[m:] == 7).all()) and bool((store[:, rows:] == 7).all())


@pytest.mark.parametrize("m,cols,group,x", [(1, 8192, 128, BF16), (16, 8192, 64, BF16), (5, 8192, 32, F32), (16, 4097, 128, F32), (7, 6000, 64, F16),
                                             (16, 8191, 32, F16), (16, 8192, 128, F32)])
def test_scores_of_wide_rows(m, cols, group, x):
    q, scales = packed(2500, cols, group)
    v = randn(m, cols, dtype=x)
    out = torch.empty((m, 2500), device="cuda")
    mb.mono_packed_scores(q, scales, group, v, out)
    check_scores(out, q, scales, group, v)


def test_scores_of_many_rows_and_behind_the_32nd_bit():
    q, scales = packed(300007, 96, 32)
    x = randn(3, 96, dtype=F16)
    out = torch.empty((3, 300007), dtype=BF16, device="cuda")
    mb.mono_packed_scores(q, scales, 32, x, out)
    check_scores(out, q, scales, 32, x)
    rows = (1 << 32) // 2048 + 100
    q = torch.full((rows, 2048), 0x88, dtype=torch.uint8, device="cuda")
    scales = torch.ones((rows, 32), dtype=F16, device="cuda")
    q[rows - 1, 2047] = 0x98
    q[(1 << 31) // 2048 + 1, 0] = 0x8A
    x = torch.ones((1, 4096), dtype=BF16, device="cuda")
    out = torch.empty((1, rows), device="cuda")
    mb.mono_packed_scores(q, scales, 128, x, out)
    assert float(out[0, rows - 1]) == 1 and float(out[0, (1 << 31) // 2048 + 1]) == 2 and float(out.abs().sum()) == 3


def test_scores_of_vectors_that_are_not_finite_stay_with_their_vector_and_their_rows():
    q, scales = packed(70, 128, 64)
    q[3] = 0x88                                            # a row of zeros
    for t in TYPES:
        x = randn(4, 128, dtype=t)
        x[1, 70], x[2, 5] = float("inf"), float("nan")
        out = torch.empty((4, 70), device="cuda")
        mb.mono_packed_scores(q, scales, 64, x, out)
        v, s = values(q, scales, 64, 128)
        check_scores(out[[0, 3]], q, scales, 64, x[[0, 3]])
        assert bool(torch.isnan(out[2]).all())
        weight = (v * s)[:, 70]
        assert torch.equal(torch.isnan(out[1]), weight == 0)
        assert torch.equal(out[1][weight != 0], torch.where(weight[weight != 0] > 0, float("inf"), float("-inf")).float())
    scales[9, 1], scales[10, 0] = float("nan"), float("inf")
    x = randn(2, 128)
    out = torch.empty((2, 70), device="cuda")
    mb.mono_packed_scores(q, scales, 64, x, out)
    assert bool(torch.isnan(out[:, 9]).all()) and bool((~torch.isfinite(out[:, 10])).all())
    out[:, 9:11] = 0
    assert bool(torch.isfinite(out).all())


def test_scores_of_large_and_small_fp32_vectors():
    q, scales = packed(100, 64, 32)
    for size in (1e-30, 1e-3, 1e30):
        x = randn(2, 64, scale=size)
        out = torch.empty((2, 100), device="cuda")
        mb.mono_packed_scores(q, scales, 32, x, out)
        check_scores(out, q, scales, 32, x)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("t", [F32, BF16])
def test_scores_whose_group_sums_are_near_the_largest_numbers(t, group):
    # every group's sum is finite in fp32: at most 8 * 32 * 2^119 = 8 * 128 * 2^117 = 2^127
    cols, top = 2 * group + 3, 118 if group == 32 else 116
    q, scales = packed(90, cols, group)
    q[3:6] = 0xFF                                          # every weight 7
    x = ((torch.rand((3, cols), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) + 1) * 2.0 ** top).to(t)
    x[1, ::2] *= -1
    # one element at the type's end, its weight 1 in row 7, -1 in row 8 and 0 elsewhere
    q[:, 0] = q[:, 0] & 0xF0 | 8
    q[7, 0], q[8, 0] = q[7, 0] & 0xF0 | 9, q[8, 0] & 0xF0 | 7
    x[2] = 0
    x[2, 0] = torch.finfo(t).max
    out = torch.empty((3, 90), device="cuda")
    mb.mono_packed_scores(q, scales, group, x, out)
    assert bool(torch.isfinite(out).all())
    check_scores(out, q, scales, group, x)


def lopsided(cols, group, k, seed=0):
    """Vectors whose columns of weight 0 (two of every quarter of a group) are 1 and the others 2^-k .. 2^(1-k), and rows for them."""
    q, scales = packed(50, cols, group, F32, seed=seed)
    q[:, ::group // 8] = 0x88
    heavy = torch.arange(cols, device="cuda") // 2 % (group // 8) == 0
    x = (1 + torch.rand((2, cols), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))) * 2.0 ** -k
    x[:, heavy] = 1.0
    return q, scales, x * torch.where(torch.arange(cols, device="cuda") % 3 == 0, -1, 1)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("t,least", [(F32, 38), (BF16, 32), (F16, 34)])
def test_scores_of_elements_that_are_small_beside_others_of_their_group(t, least, group):
    # what the large elements are multiplied by is 0, so the scores are those of the small ones, and their tolerance too
    for k in range(8, least + 1, 2):
        q, scales, x = lopsided(2 * group + 5, group, k, seed=k)
        x = (x * 2.0 ** (15 if t is F16 else -20)).to(t)      # (fp16: down to a few of its least number)
        out = torch.empty((2, 50), device="cuda")
        mb.mono_packed_scores(q, scales, group, x, out)
        check_scores(out, q, scales, group, x)


@pytest.mark.parametrize("t,least,lost", [(F32, 38, 62), (BF16, 32, 40)])
def test_scores_of_elements_that_are_smaller_than_that(t, least, lost):
    for k in range(least, lost + 6, 2):
        q, scales, x = lopsided(70, 64, k, seed=k)
        x = x.to(t)
        out = torch.empty((2, 50), device="cuda")
        mb.mono_packed_scores(q, scales, 64, x, out)
        v, s = values(q, scales, 64, 70)
        want, size = x.double() @ (v * s).T, x.double().abs() @ (v * s).abs().T
        # (the last group has one large column and five small ones; what is off by 2^-lost of the largest, 1, is every small column)
        tol = size * (64 + 2 + 16) * 2.0 ** -23 + (v * s).abs().sum(1) * 2.0 ** -lost
        assert bool(((out.double() - want).abs() <= tol).all()), k


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("top", [2.0 ** -90, 2.0 ** -100, 2.0 ** -115, 2.0 ** -124, 2.0 ** -126, 2.0 ** -130])
def test_scores_of_vectors_near_the_smallest_numbers(t, top):
    q, scales = packed(80, 100, 32, F32)
    x = (randn(3, 100).clamp(-2, 2).double() * top).to(t)
    assert bool((x != 0).any())
    out = torch.empty((3, 80), device="cuda")
    mb.mono_packed_scores(q, scales * 2.0 ** 70, 32, x, out)      # (normal numbers)
    check_scores(out, q, scales * 2.0 ** 70, 32, x)


@pytest.mark.parametrize("s", [F32, BF16])
def test_scores_of_rows_with_subnormal_scales(s):
    least = SUBNORMAL[s]
    q, _ = packed(60, 96, 32)
    scales = (torch.arange(1, 181, device="cuda").view(60, 3).double() * least).to(s)
    assert bool((scales.double() % least == 0).all()) and float(scales.double().min()) == least
    for t in (F32, BF16):                                  # (large enough that the scores are normal numbers)
        x = randn(2, 96, dtype=t, scale=2.0 ** 72)
        out = torch.empty((2, 60), device="cuda")
        mb.mono_packed_scores(q, scales, 32, x, out)
        check_scores(out, q, scales, 32, x)


def test_a_vector_alone_and_no_vectors():
    q, scales = packed(40, 64, 32)
    x, out = randn(64), torch.empty(40, device="cuda")
    mb.mono_packed_scores(q, scales, 32, x, out)
    check_scores(out[None], q, scales, 32, x[None])
    mb.mono_packed_scores(q, scales, 32, randn(3, 64)[:0], torch.empty((0, 40), device="cuda"))


def test_packed_calls_in_a_graph_and_on_another_stream():
    rows, cols = 3000, 200
    weight = randn(rows, cols)
    q, scales = packed(rows, cols, 64)
    x, tokens = randn(2, cols, dtype=BF16), some_tokens(50, rows)
    out, scores = torch.empty((50, cols), device="cuda"), torch.empty((2, rows), device="cuda")

    def step():
        mb.mono_pack_rows(weight, q, scales, 64)
        mb.mono_packed_token_rows(q, scales, 64, tokens, out)
        mb.mono_packed_scores(q, scales, 64, x, scores)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (3, 4):
        weight.copy_(randn(rows, cols, seed=seed))
        x.copy_(randn(2, cols, dtype=BF16, seed=seed))
        graph.replay()
        check_scores(scores, q, scales, 64, x)
        t = tokens.long()
        there = (t >= 0) & (t < rows)
        v, s = values(q, scales, 64, cols)
        want = torch.zeros((50, cols), dtype=torch.float64, device="cuda")
        want[there] = (v * s)[t[there]]
        assert bool(((out.double() - want).abs() <= want.abs() * 2.0 ** -23).all())
        assert bool(((v * s - weight.double()).abs() <= s * (0.5 + 2.0 ** -8)).all())
