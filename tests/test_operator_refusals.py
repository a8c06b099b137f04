"""What the operators on plain matrices refuse, before anything is enqueued: no GPU is needed (and none is touched)."""
import ctypes

import pytest
import torch

from paper_2209_07663_b200 import binding as mb

DATA = 1 << 20          # an address that nothing reads
OK_MATRIX = dict(data=DATA, rows=10, cols=64, stride=64, type=mb.MONO_F32)
OK_PACKED = dict(q=DATA, scales=DATA, rows=10, cols=64, q_stride=32, scale_stride=2, group=32, scale_type=mb.MONO_F16)


def matrix(**kw):
    return mb.mono_matrix_t(**{**OK_MATRIX, **kw})


def packed(**kw):
    return mb.mono_packed_t(**{**OK_PACKED, **kw})


def lib():
    return mb.load_library()


def rows(weight=None, out=None, tokens=DATA, type=mb.MONO_I64, n=10):
    return lib().mono_token_rows(weight or matrix(), tokens, type, n, -1, 1.0, out or matrix(), None)


def grad(grad_out=None, out=None, tokens=DATA, type=mb.MONO_I64, n=10, accumulate=0, workspace=DATA, bytes=1 << 30):
    return lib().mono_token_rows_grad(grad_out or matrix(), tokens, type, n, -1, 1.0, accumulate, out or matrix(), workspace, bytes, None)


def pack(m=None, p=None):
    return lib().mono_pack_rows(m or matrix(), p or packed(), None)


def packed_rows(p=None, out=None, tokens=DATA, type=mb.MONO_I64, n=10):
    return lib().mono_packed_token_rows(p or packed(), tokens, type, n, -1, 1.0, out or matrix(), None)


def scores(p=None, x=None, out=None):
    return lib().mono_packed_scores(p or packed(), x or matrix(rows=3), out or matrix(rows=3, cols=10, stride=10), None)


BAD_MATRIX = [dict(data=None), dict(data=DATA + 2), dict(rows=-1), dict(rows=(1 << 31) - 1), dict(cols=0), dict(cols=-4),
              dict(cols=mb.MONO_MAX_COLS + 1, stride=mb.MONO_MAX_COLS + 1), dict(stride=-64), dict(stride=(1 << 29) + 1), dict(type=3), dict(type=-1)]
BAD_WRITTEN = BAD_MATRIX + [dict(stride=63), dict(stride=0)]
BAD_PACKED = [dict(q=None), dict(q=DATA + 8), dict(scales=None), dict(scales=DATA + 1), dict(rows=-1), dict(rows=1 << 31), dict(cols=0),
              dict(cols=mb.MONO_MAX_COLS + 1), dict(q_stride=24), dict(q_stride=16), dict(q_stride=0), dict(q_stride=-32),
              dict(scale_stride=1), dict(scale_stride=-2), dict(group=0), dict(group=16), dict(group=48), dict(group=256),
              dict(scale_type=3)]


@pytest.mark.parametrize("bad", BAD_MATRIX, ids=str)
def test_matrices_that_are_read(bad):
    assert rows(weight=matrix(**bad)) == mb.MONO_ERR_ARG
    assert grad(grad_out=matrix(**bad)) == mb.MONO_ERR_ARG
    assert pack(m=matrix(**bad)) == mb.MONO_ERR_ARG
    assert scores(x=matrix(**{"rows": 3, **bad})) == mb.MONO_ERR_ARG


@pytest.mark.parametrize("bad", BAD_WRITTEN, ids=str)
def test_matrices_that_are_written(bad):
    assert rows(out=matrix(**bad)) == mb.MONO_ERR_ARG
    assert grad(out=matrix(**bad)) == mb.MONO_ERR_ARG
    assert packed_rows(out=matrix(**bad)) == mb.MONO_ERR_ARG
    if "cols" not in bad and bad.get("stride", 0) < 1 << 29:        # (a row of scores is as long as there are rows)
        assert scores(out=matrix(**{"rows": 3, "cols": 10, "stride": 10, **({**bad, "stride": 9} if bad.get("stride") == 63 else bad)})) == mb.MONO_ERR_ARG


@pytest.mark.parametrize("bad", BAD_PACKED, ids=str)
def test_packed_rows(bad):
    assert pack(p=packed(**bad)) == mb.MONO_ERR_ARG
    assert packed_rows(p=packed(**bad)) == mb.MONO_ERR_ARG
    assert scores(p=packed(**bad)) == mb.MONO_ERR_ARG


@pytest.mark.parametrize("bad", [dict(tokens=None), dict(tokens=DATA + 4), dict(type=2), dict(type=-1), dict(n=-1), dict(n=11),
                                 dict(n=(1 << 31) - 1), dict(tokens=DATA + 2, type=mb.MONO_I32)], ids=str)
def test_tokens(bad):
    for call in (rows, grad, packed_rows):
        assert call(**bad) == mb.MONO_ERR_ARG


def test_shapes_that_do_not_fit():
    assert rows(out=matrix(cols=32)) == mb.MONO_ERR_ARG
    assert rows(out=matrix(rows=9)) == mb.MONO_ERR_ARG
    assert grad(out=matrix(cols=32)) == mb.MONO_ERR_ARG
    assert grad(grad_out=matrix(rows=9)) == mb.MONO_ERR_ARG
    assert pack(m=matrix(rows=9)) == mb.MONO_ERR_ARG
    assert pack(m=matrix(cols=32)) == mb.MONO_ERR_ARG
    assert packed_rows(out=matrix(cols=32)) == mb.MONO_ERR_ARG
    assert packed_rows(out=matrix(rows=9)) == mb.MONO_ERR_ARG
    assert scores(x=matrix(rows=3, cols=32)) == mb.MONO_ERR_ARG
    assert scores(out=matrix(rows=2, cols=10)) == mb.MONO_ERR_ARG
    assert scores(out=matrix(rows=3, cols=11)) == mb.MONO_ERR_ARG


def test_null_descriptors_and_flags():
    L = lib()
    assert L.mono_token_rows(None, DATA, 1, 10, -1, 1.0, matrix(), None) == mb.MONO_ERR_ARG
    assert L.mono_token_rows(matrix(), DATA, 1, 10, -1, 1.0, None, None) == mb.MONO_ERR_ARG
    assert L.mono_token_rows_grad(None, DATA, 1, 10, -1, 1.0, 0, matrix(), DATA, 1 << 30, None) == mb.MONO_ERR_ARG
    assert L.mono_token_rows_grad(matrix(), DATA, 1, 10, -1, 1.0, 0, None, DATA, 1 << 30, None) == mb.MONO_ERR_ARG
    assert L.mono_pack_rows(None, packed(), None) == mb.MONO_ERR_ARG
    assert L.mono_pack_rows(matrix(), None, None) == mb.MONO_ERR_ARG
    assert L.mono_packed_token_rows(None, DATA, 1, 10, -1, 1.0, matrix(), None) == mb.MONO_ERR_ARG
    assert L.mono_packed_scores(None, matrix(rows=3), matrix(rows=3, cols=10), None) == mb.MONO_ERR_ARG
    assert L.mono_packed_scores(packed(), None, matrix(rows=3, cols=10), None) == mb.MONO_ERR_ARG
    assert L.mono_packed_scores(packed(), matrix(rows=3), None, None) == mb.MONO_ERR_ARG
    assert grad(accumulate=2) == mb.MONO_ERR_ARG and grad(accumulate=-1) == mb.MONO_ERR_ARG


def test_workspaces():
    for many in (1000, 10000, 1000000):
        need = mb.mono_token_rows_grad_workspace(many, 10, 64)
        assert need > 0
        sizes = dict(grad_out=matrix(rows=many), n=many)
        assert grad(bytes=need - 1, **sizes) == mb.MONO_ERR_SIZE
        assert grad(bytes=-1, **sizes) == mb.MONO_ERR_SIZE
        assert grad(workspace=None, **sizes) == mb.MONO_ERR_ARG
        assert grad(workspace=DATA + 128, **sizes) == mb.MONO_ERR_ARG
    n = ctypes.c_int64()
    for bad in ((-1, 10, 64), (10, -1, 64), (10, 10, 0), (10, 10, mb.MONO_MAX_COLS + 1), (1 << 31, 10, 64), (10, 1 << 31, 64)):
        assert lib().mono_token_rows_grad_workspace(*bad, ctypes.byref(n)) == mb.MONO_ERR_ARG
    assert lib().mono_token_rows_grad_workspace(10, 10, 64, None) == mb.MONO_ERR_ARG
    # it is enough for the largest sizes, and grows with each
    big = mb.mono_token_rows_grad_workspace((1 << 31) - 2, (1 << 31) - 2, mb.MONO_MAX_COLS)
    assert big > mb.mono_token_rows_grad_workspace(1 << 20, 1 << 20, 64) > mb.mono_token_rows_grad_workspace(1 << 10, 1 << 20, 64)
    assert mb.mono_token_rows_grad_workspace(0, 10, 64) >= 0


def test_limits_of_scores():
    assert scores(x=matrix(rows=17), out=matrix(rows=17, cols=10, stride=10)) == mb.MONO_ERR_LIMIT
    wide = dict(cols=8224, stride=8224)
    assert scores(p=packed(cols=8224, q_stride=4112, scale_stride=257), x=matrix(rows=3, **wide)) == mb.MONO_ERR_LIMIT


def test_nothing_to_do_is_no_error():
    assert rows(n=0, out=matrix(rows=0, data=None), tokens=None) == mb.MONO_OK
    assert grad(n=0, grad_out=matrix(rows=0, data=None), out=matrix(rows=0, data=None), tokens=None, workspace=DATA) == mb.MONO_OK
    assert pack(m=matrix(rows=0, data=None), p=packed(rows=0, q=None, scales=None)) == mb.MONO_OK
    assert packed_rows(n=0, out=matrix(rows=0, data=None), tokens=None) == mb.MONO_OK
    assert scores(x=matrix(rows=0, data=None), out=matrix(rows=0, cols=10, data=None)) == mb.MONO_OK


def test_struct_layouts():
    assert ctypes.sizeof(mb.mono_matrix_t) == 40
    assert ctypes.sizeof(mb.mono_packed_t) == 56


# ---- through tensors ----

def test_tensors_on_the_host_are_refused():
    w, t, o = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int64), torch.zeros(3, 8)
    q, s = torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1)
    for call in (lambda: mb.mono_token_rows(w, t, o), lambda: mb.mono_token_rows_grad(o, t, w), lambda: mb.mono_pack_rows(w, q, s, 32),
                 lambda: mb.mono_packed_token_rows(q, s, 32, t, o), lambda: mb.mono_packed_scores(q, s, 32, w, torch.zeros(4, 4))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_what_is_no_tensor_is_refused():
    for x in (None, 4096, [1, 2], "x"):
        for call in (lambda: mb.mono_token_rows(x, x, x), lambda: mb.mono_token_rows_grad(x, x, x), lambda: mb.mono_pack_rows(x, x, x, 32),
                     lambda: mb.mono_packed_token_rows(x, x, 32, x, x), lambda: mb.mono_packed_scores(x, x, 32, x, x)):
            with pytest.raises(TypeError):
                call()
    with pytest.raises(TypeError):
        mb.mono_token_rows(torch.zeros(4, 8), torch.zeros(3), torch.zeros(3, 8), scale="2")
    with pytest.raises(TypeError):
        mb.mono_token_rows(torch.zeros(4, 8), torch.zeros(3), torch.zeros(3, 8), padding=1.5)
