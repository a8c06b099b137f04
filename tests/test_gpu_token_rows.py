"""Rows by token and their gradient, against the definition in 64 bits.

Tolerances.  An element of a lookup is one product in fp32 (off by at most 2^-24 of it) rounded once to the output's type (at most
half its eps, or half the smallest subnormal).  An element of a gradient is a sum of k terms in fp32: with at most `depth` additions on
the way of any term its error is at most depth * 2^-24 * sum |term| (to first order; 2^-23 covers the rest), then a
product, perhaps one more addition, and the rounding to the output's type.  `depth` is at most k, and at most
64 (a chunk) + k / 64 / 8 (a share of the partial sums) + 2 * 8 (the shares): 128 + k / 64 is more.
"""
import itertools

import pytest
import torch

from paper_2209_07663_b200 import binding as mb

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = (F32, BF16, F16)
SUBNORMAL = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}


def randn(*shape, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def some_tokens(n, vocab, dtype=torch.int64, seed=0, strange=True, low=None, high=None):
    """Tokens, some of them outside the vocabulary."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 100)
    t = torch.randint(low or 0, high or vocab, (n,), device="cuda", generator=g)
    if strange and n > 2:
        odd = [-1, vocab, -5, 2 ** 31 - 1, -2 ** 31] + ([2 ** 40, -2 ** 63, 2 ** 63 - 1, 2 ** 32] if dtype == torch.int64 else [])
        for k, x in enumerate(odd[: max(1, n // 8)]):
            t[(7 * k + 3) % n] = x
    return t.to(dtype)


def rows64(weight, tokens, scale, padding):
    t = tokens.reshape(-1).long()
    there = (t >= 0) & (t < weight.shape[0]) & (t != padding)
    out = torch.zeros((t.numel(), weight.shape[1]), dtype=torch.float64, device="cuda")
    out[there] = weight[t[there]].double() * scale
    return out


def check_rows(got, want):
    tol = want.abs() * (torch.finfo(got.dtype).eps / 2 + 2.0 ** -23) + SUBNORMAL[got.dtype] / 2
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), f"worst {float((err - tol).max())}"
    assert bool((got[want == 0] == 0).all())


def test_no_row_is_zeros_whatever_the_factor():
    weight = randn(40, 33, dtype=BF16)
    q, scales = torch.full((40, 32), 0x12, dtype=torch.uint8, device="cuda"), torch.full((40, 2), -0.5, device="cuda")
    tokens = torch.tensor([-1, 40, 3, 7], device="cuda")
    for scale in (-1.0, float("inf"), float("nan")):
        for cols in (33, 32):
            out = torch.full((4, cols), 5.0, device="cuda")
            mb.mono_token_rows(weight[:, :cols], tokens, out, scale=scale, padding=7)
            assert bool((out[[0, 1, 3]] == 0).all()) and not bool(torch.signbit(out[[0, 1, 3]]).any())
            mb.mono_packed_token_rows(q, scales, 32, tokens, out, scale=scale, padding=7)
            assert bool((out[[0, 1, 3]] == 0).all()) and not bool(torch.signbit(out[[0, 1, 3]]).any())


def grad64(grad, tokens, vocab, scale, padding):
    t = tokens.reshape(-1).long()
    there = (t >= 0) & (t < vocab) & (t != padding)
    g = grad[there].double()
    total = torch.zeros((vocab, grad.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, t[there], g) * scale
    size = torch.zeros((vocab, grad.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, t[there], g.abs()) * abs(scale)
    count = torch.bincount(t[there], minlength=vocab)
    return total, size, count


def check_grad(got, base, grad, tokens, scale, padding, what=""):
    """base: the buffer before the call, or None where the call writes all of it."""
    total, size, count = grad64(grad, tokens, got.shape[0], scale, padding)
    want = total if base is None else total + base.double()
    depth = torch.minimum(count, 128 + count // 64)[:, None].double()
    tol = size * (depth + 4) * 2.0 ** -23 + want.abs() * (torch.finfo(got.dtype).eps / 2 + 2.0 ** -23) + SUBNORMAL[got.dtype] / 2
    met = count > 0
    err = (got.double() - want).abs()[met]
    assert bool((err <= tol[met]).all()), f"{what}: worst {float((err - tol[met]).max())}"
    left = got[~met]
    if base is None:
        assert bool((left == 0).all()), what
    else:
        assert torch.equal(left.contiguous().view(torch.uint8), base[~met].contiguous().view(torch.uint8)), what


# ---- lookup ----

@pytest.mark.parametrize("dim", [1, 2, 4, 7, 8, 12, 31, 64, 100, 257, 515, 1024, 4100])
@pytest.mark.parametrize("n", [1, 3, 65, 1000])
def test_rows_of_many_widths(n, dim):
    vocab = 300
    for k, (w, o) in enumerate(itertools.product(TYPES, TYPES)):
        weight, tokens = randn(vocab, dim, dtype=w, seed=k), some_tokens(n, vocab, (torch.int64, torch.int32)[k % 2], seed=k)
        out = torch.full((n + 2, dim), 7.0, dtype=o, device="cuda")
        mb.mono_token_rows(weight, tokens, out[:n], scale=1.7, padding=5)
        check_rows(out[:n], rows64(weight, tokens, float(torch.tensor(1.7)), 5))
        assert bool((out[n:] == 7).all())


def test_rows_as_they_are_with_a_factor_of_one():
    weight = randn(1000, 96, dtype=F16)
    weight[3, 4], weight[3, 5], weight[3, 6] = float("inf"), float("nan"), -0.0
    tokens = torch.tensor([3, 999, 0, 3], device="cuda")
    out = torch.empty((4, 96), dtype=F16, device="cuda")
    mb.mono_token_rows(weight, tokens, out)
    want = weight[tokens]
    assert torch.equal(torch.nan_to_num(out, nan=7.0), torch.nan_to_num(want, nan=7.0))
    assert bool(torch.signbit(out[0, 6]))


@pytest.mark.parametrize("w,o", [(F32, BF16), (BF16, BF16), (F16, F32)])
def test_rows_with_strides_and_odd_starts(w, o):
    vocab, n, dim = 77, 130, 64
    for start, stride in ((0, 64), (0, 72), (1, 67), (2, 66), (4, 68), (8, 96)):
        weight = randn(vocab * stride + start, dtype=w)[start:].as_strided((vocab, dim), (stride, 1))
        store = torch.full((n * stride + start + 64,), 3.0, dtype=o, device="cuda")
        out = store[start:].as_strided((n, dim), (stride, 1))
        tokens = some_tokens(n, vocab)
        mb.mono_token_rows(weight, tokens, out, scale=0.5)
        check_rows(out, rows64(weight, tokens, 0.5, -1))
        mark = torch.ones_like(store, dtype=torch.bool)
        mark[start:].as_strided((n, dim), (stride, 1))[:] = False
        assert bool((store[mark] == 3).all())


def test_rows_of_shaped_tokens_of_nothing_and_of_an_empty_vocabulary():
    weight = randn(50, 24, dtype=BF16)
    tokens = some_tokens(60, 50).view(3, 4, 5)
    out = torch.empty((3, 4, 5, 24), dtype=F32, device="cuda")
    mb.mono_token_rows(weight, tokens, out)
    check_rows(out.view(60, 24), rows64(weight, tokens, 1.0, -1))
    mb.mono_token_rows(weight, tokens.reshape(-1)[:0], out.view(60, 24)[:0])
    mb.mono_token_rows(weight[:0], tokens, out)
    assert bool((out == 0).all())


def test_rows_behind_the_32nd_bit():
    vocab, dim = (1 << 31) // 4096 + 300, 4096
    weight = torch.zeros((vocab, dim), dtype=BF16, device="cuda")
    at = torch.tensor([vocab - 1, vocab - 2, (1 << 31) // dim, 0, vocab], device="cuda")
    weight[at[:4]] = randn(4, dim, dtype=BF16)
    out = torch.empty((5, dim), dtype=BF16, device="cuda")
    mb.mono_token_rows(weight, at, out)
    check_rows(out, rows64(weight, at, 1.0, -1))


# ---- gradient ----

@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dim", [1, 2, 7, 8, 36, 64, 100, 257, 515, 1024])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 129, 255, 256, 257, 500, 512, 513, 1000, 2049, 5000, 8192, 8193])
def test_gradient_of_many_sizes(n, dim, accumulate):
    vocab = (3, 300, 1000)[n % 3]
    for k, (g, o) in enumerate(itertools.product(TYPES, TYPES)):
        grad, tokens = randn(n, dim, dtype=g, seed=k), some_tokens(n, vocab, (torch.int64, torch.int32)[k % 2], seed=k)
        before = randn(vocab, dim, dtype=o, seed=k + 50)
        got = before.clone()
        mb.mono_token_rows_grad(grad, tokens, got, scale=0.3, padding=2, accumulate=accumulate)
        check_grad(got, before if accumulate else None, grad, tokens, float(torch.tensor(0.3)), 2, f"{g} {o}")


@pytest.mark.parametrize("vocab", [1, 2, 255, 256, 511, 512, 513, 65536, 131071, 262143, 300000])
def test_gradient_of_many_vocabularies(vocab):
    # (around the digits of the sort)
    for n in (1, 77, 4096, 4097, 9000, 40000):
        grad, tokens = randn(n, 16, dtype=BF16, seed=n), some_tokens(n, vocab, torch.int64, seed=n)
        tokens[n // 2] = vocab - 1
        got = torch.full((vocab, 16), float("nan"), device="cuda")
        mb.mono_token_rows_grad(grad, tokens, got)
        check_grad(got, None, grad, tokens, 1.0, -1, f"{n}")


@pytest.mark.parametrize("n", [64, 128, 300, 512, 4096, 4160, 70000])
def test_gradient_of_one_row_and_of_rows_that_end_with_a_chunk(n):
    grad = randn(n, 72, dtype=BF16)
    for tokens in (torch.full((n,), 4, device="cuda"), torch.arange(n, device="cuda") // 64, torch.arange(n, device="cuda") // 32 % 9,
                   (torch.arange(n, device="cuda") + 1) // 128, torch.arange(n, device="cuda").flip(0) // 65):
        vocab = int(tokens.max()) + 3
        got = torch.full((vocab, 72), float("nan"), device="cuda")
        mb.mono_token_rows_grad(grad, tokens, got, scale=2.0)
        check_grad(got, None, grad, tokens, 2.0, -1)


def test_gradient_of_nothing():
    got = torch.full((40, 12), 5.0, device="cuda")
    empty = torch.empty(0, dtype=torch.int64, device="cuda")
    mb.mono_token_rows_grad(torch.empty((0, 12), device="cuda"), empty, got, accumulate=True)
    assert bool((got == 5).all())
    mb.mono_token_rows_grad(torch.empty((0, 12), device="cuda"), empty, got)
    assert bool((got == 0).all())
    # nobody's gradient is dropped, whatever it holds
    nobody = torch.full((100,), -1, device="cuda")
    bad = torch.full((100, 12), float("nan"), device="cuda")
    got.fill_(float("nan"))
    mb.mono_token_rows_grad(bad, nobody, got)
    assert bool((got == 0).all())
    got.fill_(3.0)
    mb.mono_token_rows_grad(bad, nobody, got, accumulate=True)
    assert bool((got == 3).all())
    mb.mono_token_rows_grad(bad, torch.full((100,), 7, device="cuda"), got, padding=7)
    assert bool((got == 0).all())


def test_gradient_keeps_infinities_and_nans_to_their_rows():
    grad = randn(1000, 40, dtype=F16)
    tokens = torch.arange(1000, device="cuda") % 10
    grad[13, 5], grad[24, 6], grad[34, 6] = float("nan"), float("inf"), float("-inf")
    got = torch.empty((12, 40), device="cuda")
    mb.mono_token_rows_grad(grad, tokens, got)
    nan = torch.isnan(got).nonzero().tolist()
    assert nan == [[3, 5], [4, 6]]
    assert bool(torch.isfinite(got[[0, 1, 2, 5, 6, 7, 8, 9, 10, 11]]).all())


@pytest.mark.parametrize("g,o", [(F32, F32), (BF16, F32), (BF16, BF16)])
def test_gradient_with_strides_odd_starts_and_a_broadcast_input(g, o):
    vocab, n, dim = 77, 500, 64
    tokens = some_tokens(n, vocab)
    for start, stride in ((0, 64), (0, 72), (1, 67), (2, 66), (4, 68), (8, 96)):
        grad = randn(n * stride + start, dtype=g)[start:].as_strided((n, dim), (stride, 1))
        store = torch.full((vocab * stride + start + 64,), 3.0, dtype=o, device="cuda")
        got = store[start:].as_strided((vocab, dim), (stride, 1))
        mb.mono_token_rows_grad(grad, tokens, got)
        check_grad(got, None, grad, tokens, 1.0, -1)
        mark = torch.ones_like(store, dtype=torch.bool)
        mark[start:].as_strided((vocab, dim), (stride, 1))[:] = False
        assert bool((store[mark] == 3).all())
    one = randn(1, dim, dtype=g).expand(n, dim)
    got = torch.empty((vocab, dim), dtype=o, device="cuda")
    mb.mono_token_rows_grad(one, tokens, got)
    check_grad(got, None, one, tokens, 1.0, -1)


def test_gradient_is_the_same_bits_every_time():
    n, vocab, dim = 60000, 5000, 130
    grad = randn(n, dim, dtype=BF16)
    tokens = (torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) ** 6 * vocab).long()
    outs = []
    for _ in range(5):
        got = torch.empty((vocab, dim), device="cuda")
        mb.mono_token_rows_grad(grad, tokens, got)
        outs.append(got)
    check_grad(outs[0], None, grad, tokens, 1.0, -1)
    assert all(torch.equal(outs[0], x) for x in outs[1:])


def test_gradient_is_what_differences_of_the_lookup_say():
    # the lookup is linear in the weights: <grad_out, rows(w + h) - rows(w)> = <grad, h>, exactly in 64 bits
    n, vocab, dim = 333, 40, 20
    tokens, grad, w, h = some_tokens(n, vocab), randn(n, dim), randn(vocab, dim, seed=1), randn(vocab, dim, seed=2)
    out, moved = torch.empty((n, dim), device="cuda"), torch.empty((n, dim), device="cuda")
    mb.mono_token_rows(w, tokens, out, scale=3.0, padding=1)
    mb.mono_token_rows(w + h, tokens, moved, scale=3.0, padding=1)
    got = torch.empty((vocab, dim), device="cuda")
    mb.mono_token_rows_grad(grad, tokens, got, scale=3.0, padding=1)
    left = (grad.double() * (moved.double() - out.double())).sum()
    right = (got.double() * h.double()).sum()
    # every product and every element of w + h is off by 2^-24 of itself at most
    size = (grad.double().abs() * (moved.double().abs() + out.double().abs())).sum() + (got.double().abs() * h.double().abs()).sum()
    assert abs(float(left - right)) <= float(size) * 64 * 2.0 ** -24


def test_large_gradient():
    n, vocab, dim = 300000, 50000, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = (torch.rand(n, device="cuda", generator=g) ** 8 * vocab).long()
    grad = randn(n, dim, dtype=F16, scale=0.1)
    got = torch.empty((vocab, dim), device="cuda")
    mb.mono_token_rows_grad(grad, tokens, got, padding=0)
    check_grad(got, None, grad, tokens, 1.0, 0)


def test_gradient_behind_the_32nd_bit():
    vocab, dim, n = (1 << 31) // 4096 + 300, 4096, 70
    tokens = torch.full((n,), vocab - 1, device="cuda")
    tokens[5], tokens[6] = (1 << 31) // dim + 1, 0
    grad = randn(n, dim, dtype=BF16)
    got = torch.full((vocab, dim), 1.0, dtype=BF16, device="cuda")
    mb.mono_token_rows_grad(grad, tokens, got, accumulate=True)
    at = [0, (1 << 31) // dim + 1, vocab - 1]
    total = torch.stack([grad[6].double(), grad[5].double(), grad.double().sum(0) - grad[5].double() - grad[6].double()]) + 1.0
    size = grad.double().abs().sum(0)
    assert bool(((got[at].double() - total).abs() <= size * 72 * 2.0 ** -23 + total.abs() * 2.0 ** -8).all())
    got[at] = 1.0
    assert bool((got == 1).all())
    # more rows of gradients than 32 bits count elements
    del got
    n = (1 << 31) // dim + 100
    grad = torch.zeros((n, dim), dtype=BF16, device="cuda")
    grad[n - 1], grad[n - 2] = 2.0, 1.0
    tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
    tokens[n - 2] = 1
    got = torch.empty((3, dim), device="cuda")
    mb.mono_token_rows_grad(grad, tokens, got)
    assert bool((got[0] == 2).all()) and bool((got[1] == 1).all()) and bool((got[2] == 0).all())


def test_workspace_of_the_callers_own():
    n, vocab, dim = 3000, 700, 48
    grad, tokens = randn(n, dim), some_tokens(n, vocab)
    need = mb.mono_token_rows_grad_workspace(n, vocab, dim)
    space = torch.randint(0, 256, (need + 256,), dtype=torch.uint8, device="cuda")
    got = torch.empty((vocab, dim), device="cuda")
    for _ in range(2):                                   # whatever it holds before
        mb.mono_token_rows_grad(grad, tokens, got, workspace=space[:need])
        check_grad(got, None, grad, tokens, 1.0, -1)
    with pytest.raises(mb.MonoError) as e:
        mb.mono_token_rows_grad(grad, tokens, got, workspace=space[: need - 1])
    assert e.value.code == mb.MONO_ERR_SIZE
    with pytest.raises(mb.MonoError) as e:
        mb.mono_token_rows_grad(grad, tokens, got, workspace=space[1:])
    assert e.value.code == mb.MONO_ERR_ARG


# ---- streams and graphs ----

def test_captured_calls_and_other_streams():
    n, vocab, dim = 5000, 3000, 64
    weight, tokens, grad = randn(vocab, dim, dtype=BF16), some_tokens(n, vocab), randn(n, dim, dtype=BF16)
    out, got = torch.empty((n, dim), dtype=BF16, device="cuda"), torch.empty((vocab, dim), device="cuda")

    def step():
        mb.mono_token_rows(weight, tokens, out, scale=2.0)
        mb.mono_token_rows_grad(grad, tokens, got, scale=2.0)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    check_rows(out, rows64(weight, tokens, 2.0, -1))
    check_grad(got, None, grad, tokens, 2.0, -1)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            step()
    for seed in (5, 6):
        tokens.copy_(some_tokens(n, vocab, seed=seed))
        grad.copy_(randn(n, dim, dtype=BF16, seed=seed))
        for graph in graphs:
            out.fill_(9.0), got.fill_(9.0)
            graph.replay()
            check_rows(out, rows64(weight, tokens, 2.0, -1))
            check_grad(got, None, grad, tokens, 2.0, -1)


def test_calls_at_once_on_two_streams():
    n, vocab, dim = 20000, 9000, 96
    tokens = [some_tokens(n, vocab, seed=k) for k in range(2)]
    grads = [randn(n, dim, dtype=BF16, seed=k) for k in range(2)]
    gots = [torch.empty((vocab, dim), device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                mb.mono_token_rows_grad(grads[k], tokens[k], gots[k])
    torch.cuda.synchronize()
    for k in range(2):
        check_grad(gots[k], None, grads[k], tokens[k], 1.0, -1)


# ---- sums by their depth, and what no list of marks is kept for ----

def depth_of(n, cols, count):
    """The most additions on the way of a term to its row's sum, for the rows that `count` tokens name.  Up to 512 tokens: a group's run of
    ceil(512 / groups) positions, then the pieces of the block's groups.  Beyond: a run of 8 to 64 positions, then a block's pieces (two a group at most),
    then one of each block that has the row's terms.  A group has a thread for each 8 columns, up to 32 (a power of two), a block 256 threads."""
    lanes = 1
    while lanes < 32 and lanes * 8 < -(-cols // -(-cols // 256)):
        lanes *= 2
    groups = 256 // lanes
    if n <= 512:
        return torch.clamp(count, max=-(-512 // groups) + 2 * groups)
    return torch.minimum(count, 64 + 2 * groups + 2 + count // (8 * groups))


@pytest.mark.parametrize("n,vocab", [(300, 2), (512, 1), (2049, 3), (8193, 3), (60000, 2)])
@pytest.mark.parametrize("cols", [1, 4, 8, 24, 100, 256, 515, 1024])
def test_gradient_of_rows_with_many_terms(n, vocab, cols):
    grad = randn(n, cols, dtype=BF16).abs()                # (of one sign, so that errors add up as far as they go)
    tokens = some_tokens(n, vocab, strange=False)
    got = torch.empty((vocab, cols), device="cuda")
    mb.mono_token_rows_grad(grad, tokens, got)
    total, size, count = grad64(grad, tokens, vocab, 1.0, -1)
    # each addition is off by 2^-24 of a sum of at most `size` (2^-23 covers the second order), and the product and the output as in check_grad
    tol = size * (depth_of(n, cols, count)[:, None].double() + 2) * 2.0 ** -23
    assert bool(((got.double() - total).abs() <= tol).all())


@pytest.mark.parametrize("n", [8193, 50000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_a_vocabulary_too_large_for_marks(n, accumulate):
    vocab, cols = (1 << 24) + 77, 3
    grad, tokens = randn(n, cols, dtype=BF16), some_tokens(n, vocab)
    tokens[:n // 3] = tokens[:n // 3] % 50 * (vocab // 50) + 1       # (some rows with many terms)
    tokens[5], tokens[6] = 0, vocab - 1
    before = torch.full((vocab, cols), 0.5, dtype=F16, device="cuda")
    got = before.clone()
    mb.mono_token_rows_grad(grad, tokens, got, scale=0.5, accumulate=accumulate)
    there = (tokens >= 0) & (tokens < vocab)
    rows, place = torch.unique(tokens[there], return_inverse=True)
    # the rows that tokens name, as a small vocabulary of their own, and all the others
    check_grad(got[rows], before[rows] if accumulate else None, grad[there], place, 0.5, -1)
    got[rows] = 0.5 if accumulate else 0.0
    assert bool((got == (0.5 if accumulate else 0.0)).all())


@pytest.mark.parametrize("n,vocab,cols", [(300, 7, 64), (785, 1, 1024), (1966, 32, 64), (2716, 6, 16), (2910, 5, 2048), (12921, 29, 8), (9000, 400, 264)])
@pytest.mark.parametrize("g,o", [(F32, F32), (BF16, F32), (F16, BF16)])
def test_gradient_has_the_same_bits_wherever_its_matrices_lie(n, vocab, cols, g, o):
    grad, tokens = randn(n, cols, dtype=g, seed=1), some_tokens(n, vocab, seed=2)

    def at(rows, dtype, start, stride):
        return torch.full((start + rows * stride + 8,), 3.0, dtype=dtype, device="cuda")[start:].as_strided((rows, cols), (stride, 1))

    for accumulate in (False, True):
        outs = []
        for k in (0, 1, 2, 4):
            terms, got = at(n, g, k, cols + k), at(vocab, o, 0, cols)
            terms.copy_(grad)
            mb.mono_token_rows_grad(terms, tokens, got, scale=-0.37, padding=0, accumulate=accumulate)
            far = at(vocab, o, k, cols + k)
            mb.mono_token_rows_grad(grad, tokens, far, scale=-0.37, padding=0, accumulate=accumulate)
            outs += [got.contiguous(), far.contiguous()]
        check_grad(outs[0], torch.full_like(outs[0], 3.0) if accumulate else None, grad, tokens, float(torch.tensor(-0.37)), 0)
        assert all(torch.equal(outs[0], x) for x in outs[1:])
