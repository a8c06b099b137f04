"""Rows of fixed vocabularies as torch programs use them: a differentiable lookup, and rows in 4 bits.

A feature whose vocabulary is fixed needs no hash table: its rows are a matrix and a token is a row's number.
`token_rows` is the input layer of a sequence model beside the tables' pooled features; `PackedRows` is what of a
matrix, or of a trained table's rows, goes to a serving process: looked up again, or scored against a few vectors.
Everything runs in the CUDA library (include/mono.h); there is no CPU path.  What records torch operations while they run (torch.jit.trace, make_fx)
does not see the library's: it would record the empty outputs alone.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as mb


class _TokenRows(torch.autograd.Function):
    @staticmethod
    def forward(ctx, weight, tokens, scale, padding, dtype):
        if weight.dim() != 2:
            raise ValueError("weight: a matrix of rows is expected")
        out = torch.empty((*tokens.shape, weight.shape[1]), dtype=dtype or weight.dtype, device=weight.device)
        mb.mono_token_rows(weight, tokens, out, scale=scale, padding=padding)
        ctx.save_for_backward(tokens)
        ctx.vocabulary, ctx.grad_dtype, ctx.scale, ctx.padding = weight.shape[0], weight.dtype, scale, padding
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        tokens, = ctx.saved_tensors
        cols = grad_out.shape[-1]
        grad_out = grad_out.resolve_neg().reshape(-1, cols)      # (a view, or a copy where the rows do not lie in one)
        if cols > 1 and grad_out.stride(1) != 1:
            grad_out = grad_out.contiguous()              # as a sum's gradient, which is one number everywhere
        grad_weight = torch.empty((ctx.vocabulary, cols), dtype=ctx.grad_dtype, device=grad_out.device)
        mb.mono_token_rows_grad(grad_out, tokens, grad_weight, scale=ctx.scale, padding=ctx.padding)
        return grad_weight, None, None, None, None


def token_rows(weight, tokens, scale: float = 1.0, padding: int = -1, dtype=None):
    """scale * weight[tokens], in `dtype` (None: the weight's); zeros, and no gradient, where a token is `padding` or
    outside the vocabulary.  Differentiable once with respect to `weight`; the gradient is the same bits every time.

    The gradient is a whole matrix.  A loop that adds up several steps' in a buffer of another type calls
    binding.mono_token_rows_grad(..., accumulate=True) itself, which touches the rows that tokens name alone.
    torch's rule for capturing a backward pass into a CUDA graph holds here too: while it is captured, no graph of an
    eager forward pass of the same weights may be alive.
    """
    return _TokenRows.apply(weight, tokens.contiguous(), float(scale), int(padding), dtype)


def _no_gradient(call, **tensors):
    if torch.is_grad_enabled():
        for name, x in tensors.items():
            if x is not None and x.requires_grad:
                raise RuntimeError(f"{call} has no gradient, but {name} requires one: detach it, or call under torch.no_grad()")


class PackedRows:
    """Rows in 4 bits a column with one scale per group of columns: value = (q - 8) * scale.

    For serving: nothing here has a gradient, and `rows` and `scores` refuse tensors that would need one.

    `q` is uint8 [rows, bytes], two columns in a byte (the even one in the low half), a row's bytes rounded up to a multiple
    of 16; `scales` is [rows, groups].  Both are plain tensors: a program saves, loads and moves them as it likes.
    """

    def __init__(self, q, scales, cols: int, group: int = 64):
        if group not in (32, 64, 128):
            raise ValueError("group: 32, 64 or 128 is expected")
        if q.dim() != 2 or scales.dim() != 2 or q.shape[0] != scales.shape[0]:
            raise ValueError("q and scales: matrices with as many rows are expected")
        if q.shape[1] < (cols + 31) // 32 * 16 or scales.shape[1] < -(-cols // group) or cols < 1:
            raise ValueError(f"q and scales hold no {cols} columns")
        self.q, self.scales, self.cols, self.group = q, scales, int(cols), int(group)

    @classmethod
    def empty(cls, rows: int, cols: int, group: int = 64, scale_dtype=torch.float16, device="cuda"):
        return cls(torch.empty((rows, (cols + 31) // 32 * 16), dtype=torch.uint8, device=device),
                   torch.empty((rows, -(-cols // group)), dtype=scale_dtype, device=device), cols, group)

    @classmethod
    def pack(cls, rows, group: int = 64, scale_dtype=torch.float16):
        """Of a matrix on the device.  Each column is within half a scale of what it was, a scale being a seventh of the largest
        column of its group, where scale_dtype has room for it: float16 does not for groups whose largest column is beyond 4.5e5 (NaN) or
        below 3e-6 (off by more; zeros below 2e-7), bfloat16 and float32 do."""
        p = cls.empty(rows.shape[0], rows.shape[1], group, scale_dtype, rows.device)
        mb.mono_pack_rows(rows, p.q, p.scales, group)
        return p

    def __len__(self):
        return self.q.shape[0]

    def replace(self, at, rows):
        """Pack `rows` in the place of those at `at`: what a serving process does with the rows that MonoTable.export_touched
        shipped.  at: int64, distinct row numbers from 0 on, which is checked (and waited for), but not while a CUDA graph is captured."""
        if rows.dim() != 2 or rows.shape[1] != self.cols:
            raise ValueError(f"rows: a matrix of {self.cols} columns is expected")
        if at.dim() != 1 or at.shape[0] != rows.shape[0]:
            raise ValueError("at: a row number for each of the rows is expected")
        if at.dtype != torch.int64 or at.device != self.q.device:
            raise ValueError("at: int64 row numbers on the packed rows' device are expected")
        if at.numel() and not torch.cuda.is_current_stream_capturing():
            # a number outside would end the context in a device assertion, a repeated one mix one row's columns with another's scales
            ordered = at.sort().values
            if bool((ordered[0] < 0) | (ordered[-1] >= len(self)) | (ordered[1:] == ordered[:-1]).any()):
                raise ValueError(f"at: distinct row numbers below {len(self)} are expected")
        p = PackedRows.pack(rows, self.group, self.scales.dtype)
        self.q[:, :p.q.shape[1]].index_copy_(0, at, p.q)
        self.scales[:, :p.scales.shape[1]].index_copy_(0, at, p.scales)

    def rows(self, tokens, scale: float = 1.0, padding: int = -1, dtype=torch.float32, out=None):
        """scale * the rows that `tokens` name; zeros where a token is `padding` or names none."""
        _no_gradient("rows", out=out, scales=self.scales)
        tokens = tokens.contiguous()
        if out is None:
            out = torch.empty((*tokens.shape, self.cols), dtype=dtype, device=self.q.device)
        elif out.shape[-1] != self.cols:
            raise ValueError(f"out: {self.cols} columns are expected")
        mb.mono_packed_token_rows(self.q, self.scales, self.group, tokens, out, scale=scale, padding=padding)
        return out

    def scores(self, x, dtype=torch.float32, out=None):
        """<x, row> for every row: [rows] of one vector, [vectors, rows] of up to binding.MONO_MAX_SCORED."""
        _no_gradient("scores", x=x, out=out, scales=self.scales)
        if x.shape[-1] != self.cols:
            raise ValueError(f"x: {self.cols} columns are expected")
        if out is None:
            out = torch.empty((*x.shape[:-1], len(self)), dtype=dtype, device=self.q.device)
        mb.mono_packed_scores(self.q, self.scales, self.group, x, out)
        return out
