"""The torch side of fixed vocabularies: the differentiable lookup, packed rows, and both beside a table."""
import numpy as np
import pytest
import torch

import paper_2209_07663_b200 as pkg
from paper_2209_07663_b200 import binding as mb
from paper_2209_07663_b200 import workload as wl
from paper_2209_07663_b200.tokens import PackedRows, token_rows
from tests.test_gpu_packed_rows import check_scores, values
from tests.test_gpu_token_rows import BF16, F16, F32, check_grad, check_rows, randn, rows64, some_tokens

pytestmark = pytest.mark.gpu


def test_they_are_what_the_package_offers():
    assert pkg.token_rows is token_rows and pkg.PackedRows is PackedRows
    with pytest.raises(AttributeError):
        pkg.no_such_name


@pytest.mark.parametrize("dtype,out", [(F32, None), (BF16, None), (F32, BF16), (F16, F32)])
def test_gradients_of_a_small_model(dtype, out):
    weight = randn(300, 48, dtype=dtype).requires_grad_()
    tokens = some_tokens(4 * 33, 300).view(4, 33)
    head = randn(48, 5, seed=1)
    rows = token_rows(weight, tokens, scale=2.5, padding=7, dtype=out)
    assert rows.dtype == (out or dtype) and rows.shape == (4, 33, 48)
    check_rows(rows.detach().view(-1, 48), rows64(weight.detach(), tokens, 2.5, 7))
    (rows.float() @ head).square().sum().backward()
    grad_rows = (2 * (rows.detach().float() @ head) @ head.T).to(rows.dtype).view(-1, 48)
    assert weight.grad.dtype == dtype
    # the gradient that reached the lookup is rounded to the rows' type; what torch's own products lose is below it
    total_of = grad_rows.double().abs()
    check = weight.grad.double()
    t = tokens.reshape(-1)
    there = (t >= 0) & (t < 300) & (t != 7)
    want = torch.zeros((300, 48), dtype=torch.float64, device="cuda").index_add_(0, t[there], grad_rows[there].double()) * 2.5
    size = torch.zeros((300, 48), dtype=torch.float64, device="cuda").index_add_(0, t[there], total_of[there]) * 2.5
    # products of 5 and of 48 terms in fp32, taken here in another order than in the model, and one rounding on each side
    slack = size * (2.0 ** -16 + torch.finfo(rows.dtype).eps) + want.abs() * torch.finfo(dtype).eps / 2
    assert bool(((check - want).abs() <= slack + 1e-6 * size.max()).all())


@pytest.mark.parametrize("what", ["sum", "slice", "transposed", "one column"])
def test_gradients_that_do_not_lie_in_rows(what):
    cols = 1 if what == "one column" else 24
    weight = randn(50, cols).requires_grad_()
    tokens = some_tokens(60, 50).view(6, 10)
    rows = token_rows(weight, tokens)
    if what in ("sum", "one column"):
        rows.sum().backward()
        grad = torch.ones(60, cols, device="cuda")
    elif what == "slice":
        pick = randn(6, 10, 12, seed=2)
        (rows[..., ::2] * pick).sum().backward()
        grad = torch.zeros(6, 10, 24, device="cuda")
        grad[..., ::2] = pick
        grad = grad.view(60, 24)
    else:
        pick = randn(24, 6, 10, seed=3)
        (rows.permute(2, 0, 1) * pick).sum().backward()
        grad = pick.permute(1, 2, 0).reshape(60, 24)
    check_grad(weight.grad, None, grad, tokens, 1.0, -1)


def test_the_gradient_agrees_with_differences():
    weight = randn(20, 6).double()
    tokens = some_tokens(40, 20)
    pick = randn(40, 6, seed=4)
    w = weight.float().requires_grad_()
    (token_rows(w, tokens, scale=0.5, padding=3) * pick).sum().backward()
    step = 2.0 ** -3                         # a power of two: the lookup is linear, so a large step loses nothing
    for r, c in ((0, 0), (3, 2), (7, 5), (19, 1)):
        moved = weight.float().clone()
        moved[r, c] += step
        up = (token_rows(moved, tokens, scale=0.5, padding=3).double() * pick.double()).sum()
        moved[r, c] -= 2 * step
        down = (token_rows(moved, tokens, scale=0.5, padding=3).double() * pick.double()).sum()
        # the elements moved are rounded to fp32 once on each side: 2^-24 of at most (|w| + step) * |pick| * count
        size = 40 * (float(weight.abs().max()) + 1) * float(pick.abs().max())
        assert abs(float((up - down) / (2 * step)) - float(w.grad[r, c])) <= size * 2.0 ** -20


def test_shared_weights_and_several_lookups_add_up():
    weight = randn(40, 16).requires_grad_()
    a, b = some_tokens(30, 40, seed=1), some_tokens(50, 40, seed=2)
    (token_rows(weight, a, scale=2.0).sum() + token_rows(weight, b, scale=3.0).sum()).backward()
    tokens = torch.cat((a, b))
    grad = torch.cat((torch.full((30, 16), 2.0, device="cuda"), torch.full((50, 16), 3.0, device="cuda")))
    check_grad(weight.grad, None, grad, tokens, 1.0, -1)
    with pytest.raises(RuntimeError):        # differentiable once
        out = token_rows(weight, a)
        g, = torch.autograd.grad(out.square().sum(), weight, create_graph=True)
        g.sum().backward()


def test_a_written_output_is_noticed_by_autograd():
    w = randn(10, 8)
    out = torch.ones(4, 8, device="cuda", requires_grad=True) * 2
    y = out.square().sum()
    mb.mono_token_rows(w, torch.zeros(4, dtype=torch.int64, device="cuda"), out.detach())
    with pytest.raises(RuntimeError, match="modified"):
        y.backward()
    with torch.inference_mode():
        mb.mono_token_rows(w, torch.zeros(4, dtype=torch.int64, device="cuda"), torch.empty(4, 8, device="cuda"))


def test_a_captured_step():
    tokens = some_tokens(500, 200).view(5, 100)
    weight = randn(200, 32, dtype=BF16).requires_grad_()
    pick = randn(5, 100, 32, dtype=BF16, seed=5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            weight.grad = None
            (token_rows(weight, tokens, scale=2.0) * pick).sum().backward()
    torch.cuda.current_stream().wait_stream(side)
    weight.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        (token_rows(weight, tokens, scale=2.0) * pick).sum().backward()
    for seed in (7, 8):
        pick.copy_(randn(5, 100, 32, dtype=BF16, seed=seed))
        graph.replay()
        check_grad(weight.grad, None, pick.view(500, 32), tokens, 2.0, -1)


def test_tensors_that_are_refused():
    w, t, o = randn(10, 8), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.empty(4, 8, device="cuda")
    for call, error in [
        (lambda: mb.mono_token_rows(w.double(), t, o), TypeError),
        (lambda: mb.mono_token_rows(w.long(), t, o), TypeError),
        (lambda: mb.mono_token_rows(w, t.short(), o), TypeError),
        (lambda: mb.mono_token_rows(w, t.float(), o), TypeError),
        (lambda: mb.mono_token_rows(w.t(), t, o), ValueError),
        (lambda: mb.mono_token_rows(w, torch.zeros(8, dtype=torch.int64, device="cuda")[::2], o), ValueError),
        (lambda: mb.mono_token_rows(w, t.cpu(), o), ValueError),
        (lambda: mb.mono_token_rows(w.cpu(), t, o), ValueError),
        (lambda: mb.mono_token_rows(w, t, o[:, :4].contiguous()), mb.MonoError),
        (lambda: mb.mono_token_rows(w, t, o[:3]), mb.MonoError),
        (lambda: mb.mono_token_rows(w, t, o[:1].expand(4, 8)), mb.MonoError),
        (lambda: mb.mono_token_rows(w, t, torch.tensor(1.0, device="cuda")), ValueError),
        (lambda: mb.mono_token_rows_grad(o, t, w[:1].expand(10, 8)), mb.MonoError),
        (lambda: mb.mono_token_rows_grad(o, t, w, workspace=torch.empty(8, 64, device="cuda").t()), ValueError),
        (lambda: token_rows(w[0], t), ValueError),
    ]:
        with pytest.raises(error):
            call()
    p = PackedRows.pack(w, 32)
    for call, error in [
        (lambda: PackedRows.pack(w, 48), ValueError),
        (lambda: PackedRows(p.q, p.scales, 33, 32), ValueError),
        (lambda: PackedRows(p.q[:5], p.scales, 8, 32), ValueError),
        (lambda: p.scores(randn(3, 9)), ValueError),
        (lambda: p.rows(t, out=torch.empty(4, 9, device="cuda")), ValueError),
        (lambda: p.scores(randn(17, 8)), mb.MonoError),
        (lambda: p.scores(randn(8).double()), TypeError),
        (lambda: mb.mono_packed_scores(p.q, p.scales, 48, randn(1, 8), torch.empty(1, 10, device="cuda")), ValueError),
        (lambda: mb.mono_packed_scores(p.q.char(), p.scales, 32, randn(1, 8), torch.empty(1, 10, device="cuda")), TypeError),
        (lambda: mb.mono_packed_scores(p.q, p.scales[:9], 32, randn(1, 8), torch.empty(1, 10, device="cuda")), ValueError),
        (lambda: mb.mono_packed_scores(p.q, p.scales, 32, randn(1, 64), torch.empty(1, 10, device="cuda")), ValueError),
        (lambda: mb.mono_packed_scores(p.q[:, ::2], p.scales, 32, randn(1, 8), torch.empty(1, 10, device="cuda")), ValueError),
        (lambda: mb.mono_pack_rows(w, p.q[:9], p.scales[:9], 32), mb.MonoError),
    ]:
        with pytest.raises(error):
            call()
    with torch.device("cuda"):               # a torch function mode: tensors are read as they are
        mb.mono_token_rows(w, t, o)
        assert p.scores(randn(8)).shape == (10,)


def test_a_table_and_a_vocabulary_trained_served_and_scored():
    """Pooled features from a table and tokens from a matrix, trained together; then the table's rows in 4 bits."""
    cfg = wl.scaled(wl.CONFIGS["tiny"], n_examples=64, steps=6)
    table = mb.MonoTable(cfg.capacity, cfg.dim, 1, 0, lr=0.1, init_scale=0.5, seed=3)
    vocabulary = randn(100, cfg.dim, seed=1)
    total = torch.zeros_like(vocabulary)
    stream = wl.Stream(cfg)
    for step in range(cfg.steps):
        s = stream.step(step)
        pooled = table.lookup_pool(s.ids, s.offsets)
        tokens = some_tokens(pooled.shape[0], 100, seed=step)
        rows = token_rows(vocabulary, tokens, scale=0.5)
        mix = pooled + rows                                  # a loss of <mix, mix> / 2
        table.apply_grads(s.ids, s.offsets, mix, step)
        before = total.clone()
        mb.mono_token_rows_grad(mix, tokens, total, scale=0.5, accumulate=True)
        check_grad(total, before, mix, tokens, 0.5, -1)
    ids, packed = table.export_packed(group=32, scale_dtype=F32)
    state = table.export()
    own = state["resident"] == 1
    by_bits = np.argsort(state["ids"][own].view(np.int64), kind="stable")
    assert np.array_equal(ids.cpu().numpy(), state["ids"][own].view(np.int64)[by_bits])
    w = torch.from_numpy(state["w"][own][by_bits]).cuda()
    assert len(packed) == w.shape[0] > 1000 and packed.cols == cfg.dim
    back = packed.rows(torch.arange(len(packed), device="cuda"))
    scale = packed.scales.repeat_interleave(32, 1)[:, :cfg.dim]
    # half a step of the rounding, and what the quotient and the product lose
    assert bool(((back - w).abs() <= scale * (0.5 + 2.0 ** -20)).all())
    users = randn(3, cfg.dim, seed=9)
    got = packed.scores(users)
    check_scores(got, packed.q, packed.scales, 32, users)
    assert packed.scores(users[0]).shape == (len(packed),)
    # the rows that were trained since the export replace those of the serving side
    table.export_touched()
    s = stream.step(1)
    table.apply_grads(s.ids, s.offsets, torch.ones((cfg.n_bags, cfg.dim), device="cuda"), cfg.steps)
    touched = table.export_touched()
    at = torch.searchsorted(ids, torch.from_numpy(touched["ids"].view(np.int64)).cuda())
    packed.replace(at, torch.from_numpy(touched["w"]).cuda())
    ids2, again = table.export_packed(group=32, scale_dtype=F32)
    assert torch.equal(ids, ids2) and torch.equal(packed.q, again.q) and torch.equal(packed.scales, again.scales)
    v, f = values(packed.q, packed.scales, 32, cfg.dim)
    assert bool((packed.rows(at[:5]).double() == (v * f)[at[:5]].float().double()).all())
    table.close()


def test_a_table_without_rows_exports_none():
    table = mb.MonoTable(1024, 16, 2, 0)
    ids, packed = table.export_packed(group=128)
    assert ids.numel() == 0 and len(packed) == 0
    assert packed.scores(randn(2, 16)).shape == (2, 0)
    assert bool((packed.rows(torch.arange(5, device="cuda")) == 0).all())
    # tracked, but below the threshold
    one = torch.arange(1, 9, device="cuda")
    table.apply_grads(one, torch.arange(9, device="cuda"), torch.ones((8, 16), device="cuda"), 1)
    assert table.export_packed()[0].numel() == 0
    table.apply_grads(one[:3], torch.arange(4, device="cuda"), torch.ones((3, 16), device="cuda"), 2)
    ids, packed = table.export_packed()
    assert ids.tolist() == [1, 2, 3] and len(packed) == 3
    table.close()


@pytest.mark.parametrize("cols,group,others", [(64, 32, (32, 63, 65, 128)), (40, 32, (8, 33, 41, 64, 72)), (130, 128, (1, 128, 131, 160))])
def test_rows_of_another_width_replace_none(cols, group, others):
    packed = PackedRows.pack(randn(10, cols), group)
    q, scales, at = packed.q.clone(), packed.scales.clone(), torch.tensor([3, 7], device="cuda")
    for rows, to in [(randn(2, c), at) for c in others] + [(randn(2, cols), at[:1]), (randn(3, cols), at), (randn(2, cols), at[:, None]), (randn(cols), at[:1])]:
        with pytest.raises(ValueError):
            packed.replace(to, rows)
    assert torch.equal(packed.q, q) and torch.equal(packed.scales, scales)
    new = randn(2, cols, seed=1)
    packed.replace(at, new)
    want = PackedRows.pack(new, group)
    assert torch.equal(packed.q[at], want.q) and torch.equal(packed.scales[at], want.scales)
    rest = [r for r in range(10) if r not in (3, 7)]
    assert torch.equal(packed.q[rest], q[rest]) and torch.equal(packed.scales[rest], scales[rest])
    packed.replace(at[:0], new[:0])


def test_row_numbers_that_name_no_row_or_one_twice_replace_none():
    packed = PackedRows.pack(randn(10, 64), 32)
    q, scales, new = packed.q.clone(), packed.scales.clone(), randn(3, 64, seed=1)
    for at in ([0, 1, 10], [0, -1, 2], [3, 4, 3], [-1, -1, -1], [2 ** 40, 1, 2], [-2 ** 63, 2 ** 63 - 1, 0]):
        with pytest.raises(ValueError):
            packed.replace(torch.tensor(at, device="cuda"), new)
    for at in (torch.arange(3, device="cuda", dtype=torch.int32), torch.arange(3), torch.zeros(3, device="cuda")):
        with pytest.raises(ValueError):
            packed.replace(at, new)
    with pytest.raises(ValueError):
        PackedRows.empty(0, 64, 32).replace(torch.zeros(1, dtype=torch.int64, device="cuda"), new[:1])
    assert torch.equal(packed.q, q) and torch.equal(packed.scales, scales)
    packed.replace(torch.tensor([9, 0, 5], device="cuda"), new)
    want = PackedRows.pack(new, 32)
    assert torch.equal(packed.q[[9, 0, 5]], want.q) and torch.equal(packed.scales[[9, 0, 5]], want.scales)


def test_rows_are_replaced_in_a_graph():
    packed = PackedRows.pack(randn(10, 64), 32)
    at, new = torch.tensor([4, 2], device="cuda"), randn(2, 64, seed=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        packed.replace(at, new)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        packed.replace(at, new)
    at.copy_(torch.tensor([7, 0], device="cuda"))
    new.copy_(randn(2, 64, seed=2))
    graph.replay()
    want = PackedRows.pack(new, 32)
    assert torch.equal(packed.q[[7, 0]], want.q) and torch.equal(packed.scales[[7, 0]], want.scales)


@pytest.mark.parametrize("stream", ["its own", "another"])
def test_an_export_has_no_more_fp32_rows_at_once_than_it_says(stream, monkeypatch):
    tracked, owners, dim = 1 << 19, 5000, 512
    table = mb.MonoTable(1 << 16, dim, 2, 0, key_cells=1 << 20, lr=0.1, init_scale=0.5, seed=1)
    ids = torch.randperm(tracked, device="cuda") + 1
    bag = torch.zeros(1, dim, device="cuda")
    for part in (*ids.split(1 << 16), ids[:owners]):           # the first pass counts them, the second gives some a row
        table.apply_grads(part, torch.tensor([0, part.numel()], device="cuda"), bag, 1)
    want = table.probe(ids[:owners].sort().values)["w"]
    monkeypatch.setattr(mb.MonoTable, "PACK_BYTES", 4 * dim * 1024 + 100)      # (1024 rows, five times)
    torch.cuda.synchronize()
    other = torch.cuda.current_stream() if stream == "its own" else torch.cuda.Stream()
    with torch.cuda.stream(other):
        torch.cuda.empty_cache()
        if stream == "another":                                 # memory that is free again, but for work that is under way
            busy = torch.empty(1 << 24, device="cuda")
            for _ in range(200):
                busy.fill_(7.0)
            del busy
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        got, packed = table.export_packed(group=32, scale_dtype=F32)
    other.synchronize()
    taken = torch.cuda.max_memory_allocated() - before
    # the buffer, the packed rows (dim / 2 + 4 * dim / 32 bytes each), and up to ten 64-bit numbers for each ID
    assert taken < 4 * dim * 1024 + owners * (dim // 2 + dim // 8) + 80 * tracked < 4 * dim * tracked // 16
    assert torch.equal(got, ids[:owners].sort().values) and len(packed) == owners
    again = PackedRows.pack(torch.from_numpy(want).cuda(), 32, F32)
    assert torch.equal(packed.q, again.q) and torch.equal(packed.scales, again.scales)
    monkeypatch.setattr(mb.MonoTable, "PACK_BYTES", 1)         # a row at a time
    assert torch.equal(table.export_packed(group=32, scale_dtype=F32)[1].q, again.q)
    table.close()


def test_a_refused_call_leaves_an_outputs_version_alone():
    w, t, o = randn(10, 8), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.empty(4, 8, device="cuda")
    p = PackedRows.pack(w, 32)
    refused = [
        (o, lambda: mb.mono_token_rows(w, t[:3], o)),
        (o, lambda: mb.mono_token_rows(w, t.cpu(), o)),
        (w, lambda: mb.mono_token_rows_grad(o, t[:3], w)),
        (w, lambda: mb.mono_token_rows_grad(o.repeat(200, 1), t.repeat(200), w, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))),
        (w, lambda: mb.mono_token_rows_grad(o, t, w, workspace=1)),
        (p.q, lambda: mb.mono_pack_rows(w[:5], p.q, p.scales, 32)),
        (p.scales, lambda: mb.mono_pack_rows(w[:5], p.q, p.scales, 32)),
        (o, lambda: mb.mono_packed_token_rows(p.q, p.scales, 32, t[:3], o)),
        (o, lambda: mb.mono_packed_token_rows(p.q, p.scales, 48, t, o)),
        (o, lambda: mb.mono_packed_scores(p.q, p.scales, 32, randn(4, 8), o)),
        (o, lambda: mb.mono_packed_scores(p.q, p.scales, 32, randn(17, 8), o)),
    ]
    for written, call in refused:
        version = written._version
        with pytest.raises((mb.MonoError, ValueError, TypeError)):
            call()
        assert written._version == version
    x = torch.ones(4, 8, device="cuda", requires_grad=True) * 2
    y = x.square().sum()
    with pytest.raises(mb.MonoError):
        mb.mono_token_rows(w, t[:3], x.detach())
    y.backward()                                           # (what was not written is not "modified")
    made = torch.empty(1, 10, device="cuda")
    for written, call in [(o, lambda: mb.mono_token_rows(w, t, o)), (w, lambda: mb.mono_token_rows_grad(o, t, w)),
                          (p.q, lambda: mb.mono_pack_rows(w, p.q, p.scales, 32)), (p.scales, lambda: mb.mono_pack_rows(w, p.q, p.scales, 32)),
                          (o, lambda: mb.mono_packed_token_rows(p.q, p.scales, 32, t, o)),
                          (made, lambda: mb.mono_packed_scores(p.q, p.scales, 32, randn(1, 8), made))]:
        version = written._version
        call()
        assert written._version == version + 1


def test_packed_rows_refuse_what_would_need_a_gradient():
    p, t = PackedRows.pack(randn(10, 8).requires_grad_(), 32), torch.arange(3, device="cuda")      # (packing is of the values)
    x, leaf, made = randn(2, 8).requires_grad_(), torch.zeros(3, 8, device="cuda", requires_grad=True), torch.zeros(2, 10, device="cuda").requires_grad_()
    learned = PackedRows(p.q, p.scales.float().requires_grad_(), 8, 32)
    calls = [lambda: p.scores(x), lambda: p.scores(x * 2), lambda: p.scores(x.detach(), out=made), lambda: p.rows(t, out=leaf), lambda: p.rows(t, out=leaf * 2),
             lambda: learned.rows(t), lambda: learned.scores(x.detach())]
    for call in calls:
        with pytest.raises(RuntimeError, match="no gradient"):
            call()
    assert bool((leaf == 0).all()) and bool((made == 0).all())
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            assert torch.equal(p.scores(x), p.scores(x.detach()))
            assert torch.equal(learned.scores(x), p.scores(x))
            p.rows(t, out=leaf.detach())
    assert torch.equal(leaf.detach(), p.rows(t))
    assert p.scores(x.detach()).shape == (2, 10)


def test_scores_of_no_packed_rows():
    p = PackedRows.pack(randn(5, 16)[:0], 32)
    for shape in ((16,), (1, 16), (3, 16), (2, 3, 16), (0, 16), (2, 0, 16), (1, 1, 16)):
        assert p.scores(randn(*shape)).shape == (*shape[:-1], 0)
    mb.mono_packed_scores(p.q, p.scales, 32, randn(16), torch.empty(0, device="cuda"))
    for x, out in ((randn(2, 16), torch.empty(0, device="cuda")), (randn(16), torch.empty(2, 0, device="cuda"))):
        with pytest.raises(mb.MonoError):
            mb.mono_packed_scores(p.q, p.scales, 32, x, out)
    # where rows are looked up, they have columns
    with pytest.raises(mb.MonoError):
        mb.mono_token_rows(randn(4, 0), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"))


def test_views_that_negate_their_memory_are_refused():
    w = torch.complex(randn(5, 1), randn(5, 1, seed=2)).conj().imag        # (one column: its rows are two elements apart)
    assert w.is_neg()
    t, out = torch.arange(3, device="cuda"), torch.empty(3, 1, device="cuda")
    packed = PackedRows.pack(randn(3, 1), 32)
    for call in (lambda: mb.mono_token_rows(w, t, out), lambda: mb.mono_token_rows_grad(out, t, w), lambda: mb.mono_token_rows(out, t, w[:3]),
                 lambda: PackedRows.pack(w), lambda: packed.scores(w)):
        with pytest.raises(ValueError, match="resolve_neg"):
            call()
    mb.mono_token_rows(w.resolve_neg(), t, out)
    assert torch.equal(out, w[:3].clone())


@pytest.mark.parametrize("cols", [1, 6])
def test_gradients_that_are_such_views(cols):
    weight, tokens, other = randn(9, cols).requires_grad_(), torch.arange(20, device="cuda") % 9, randn(20, cols, seed=1)
    pick = randn(20, cols, seed=2)
    rows = token_rows(weight, tokens)
    seen = []
    rows.register_hook(lambda g: seen.append(g.is_neg()))
    z = torch.complex(other, pick)
    rows.backward(z.conj().imag)
    assert seen == [True]
    check_grad(weight.grad, None, -pick, tokens, 1.0, -1)
