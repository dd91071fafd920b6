"""Binding for include/experts_fp8.h: block-scaled 8-bit floating-point products, and routing to experts around them.

Same names and manner as `binding`: arguments are marshalled, nothing is computed here; results are new tensors for the call's
stream, or the caller's (`out`); a call the library refuses raises `binding.ConvError`, a tensor of the wrong type or shape
TypeError or ValueError.  Matrices are row-major with neighbouring elements in a row; rows may lie further apart.  New 8-bit
results have rows that begin on 16 bytes (the distance of two rows is a multiple of 16), which is what the products read fastest.

Gradients are calls of their own (`..._backward`, `gemm_fp8_experts_grad`, and for the products the products themselves); autograd records none of these calls.  A tensor
that requires a gradient is refused with ValueError while autograd records: call under `torch.no_grad()`, or in the forward and backward of an `autograd.Function`.
"""
from __future__ import annotations

import torch

from . import binding

FORMS = {"rows": 0, "columns": 1, "rows+columns": 2, "tiles": 3, "tiles_t": 4}
SCORES = {"softmax": False, "sigmoid": True}

EXPORTS = [
    "quantize_fp8_rows", "quantize_fp8_columns", "quantize_fp8_tiles", "silu_gate_backward", "gemm_fp8_nt", "gemm_fp8_experts",
    "gemm_fp8_experts_grad", "route_experts", "route_experts_backward", "expert_rows_capacity", "expert_rows", "combine_experts",
    "combine_experts_backward",
]

_native = None


def _calls():
    global _native
    if _native is None:
        _native = binding._calls()
    return _native


def _of(table, key, what):
    try:
        return table[key]
    except (KeyError, TypeError):
        raise ValueError(f"{what} must be one of {', '.join(map(repr, table))}, not {key!r}") from None


def quantize_fp8(x: torch.Tensor, form="rows", gate=False, rows=None, per_row=1, out=None, stream=None):
    """(e4m3 values, f32 scales) with a power-of-two scale for each 128 values.

    form "rows"          values [M, K], scales [ceil(K/128), M]: left operands of the products
         "columns"       of x transposed: values [K, M], scales [ceil(M/128), K]: both operands of a weights' gradient
         "rows+columns"  both, from one read of x: four tensors
         "tiles"         a scale for 128 x 128 (weights, [N, K] or [E, N, K]): scales [..., ceil(N/128), ceil(K/128)]
         "tiles_t"       the same of the transposed matrices (weights of an input's gradient)
    gate: of silu(first half of the columns) * (second half).  rows: int32 vector; row r is x[rows[r] // per_row], zeros
    where rows[r] is negative (the order of `expert_rows`)."""
    return (_native or _calls()).quantize_fp8(x, _of(FORMS, form, "form"), gate, rows, per_row, out, stream)


def silu_gate_backward(x: torch.Tensor, dh: torch.Tensor, out=None, stream=None):
    """Gradient of silu(g) * u: x [M, 2 K] holds g and u, dh [M, K] -> [M, 2 K]."""
    return (_native or _calls()).silu_gate_backward(x, dh, out, stream)


def gemm_fp8_nt(a, a_scale, b, b_scale, b_rows=False, dtype=torch.bfloat16, fast_sums=False, out=None, stream=None):
    """a [M, K] times b [N, K] transposed -> [M, N].  a_scale [ceil(K/128), M]; b_scale [ceil(N/128), ceil(K/128)], with
    b_rows [ceil(K/128), N].  fast_sums: a block's 128 products may be summed by the 8-bit matrix instruction, up to twice as fast, which
    cuts each of eight neighbouring products towards zero to a multiple of 2^-13 of the largest one's power of two: off by up to 8.5e-4 of the sum of the terms'
    magnitudes, in the mean of values of one size 1.5e-5 of the result (a hundredth of rounding to bfloat16); else in 32 bits throughout."""
    return (_native or _calls()).gemm_fp8_nt(a, a_scale, b, b_scale, b_rows, dtype, fast_sums, out, stream)


def gemm_fp8_experts(a, a_scale, w, w_scale, offsets, rows=None, per_row=1, dtype=torch.bfloat16, fast_sums=False, out=None, stream=None):
    """Rows offsets[e] ... offsets[e + 1] - 1 of the result are products with w[e] ([E, N, K], scales [E, ceil(N/128), ceil(K/128)]):
    of a's same row, or with `rows` of a's row rows[r] // per_row; zeros where there is none."""
    return (_native or _calls()).gemm_fp8_experts(a, a_scale, w, w_scale, offsets, rows, per_row, dtype, fast_sums, out, stream)


def gemm_fp8_experts_grad(a, a_scale, b, b_scale, offsets, dtype=torch.float32, fast_sums=False, out=None, stream=None):
    """a [N, R], b [K, R] (quantised by columns) -> [E, N, K]: for each expert the product over its rows offsets[e] ... offsets[e + 1] - 1."""
    return (_native or _calls()).gemm_fp8_experts_grad(a, a_scale, b, b_scale, offsets, dtype, fast_sums, out, stream)


def route_experts(logits, k, score="softmax", bias=None, groups=1, kept=1, group_top=1, renormalise=True, factor=1.0, out=None, stream=None):
    """(ids [T, k] int32, weights [T, k] f32) of each token's k experts in falling order of score + bias, among the `kept` of `groups`
    groups whose group_top largest sum to most; ties go to the lower index; -1 and 0 where fewer are to be had (logits of -infinity
    or NaN)."""
    return (_native or _calls()).route_experts(logits, k, _of(SCORES, score, "score"), bias, groups, kept, group_top, renormalise, factor, out, stream)


def route_experts_backward(dweights, ids, logits, score="softmax", renormalise=True, factor=1.0, out=None, stream=None):
    """Gradient of the logits from that of route_experts' weights."""
    return (_native or _calls()).route_experts_backward(dweights, ids, logits, _of(SCORES, score, "score"), renormalise, factor, out, stream)


def expert_rows(ids, experts, align=1, out=None, stream=None):
    """(offsets [experts + 1], rows [R], place, ids' shape) int32: the pairs (token, choice) in the experts' order.  rows: the pair of a row,
    -1 where there is none; place: the row of a pair, -1 for an id that is no expert.  Every offset is a multiple of `align`."""
    return (_native or _calls()).expert_rows(ids, experts, align, out, stream)


def combine_experts(y, place, weights=None, out=None, stream=None):
    """Each token's sum of weights[t, j] * y[place[t, j]]; without weights of the rows themselves (an input's gradient)."""
    return (_native or _calls()).combine_experts(y, place, weights, out, stream)


def combine_experts_backward(dout, y, place, rows, weights=None, out=None, stream=None):
    """(gradient of y, gradient of the weights)."""
    return (_native or _calls()).combine_experts_backward(dout, y, place, rows, weights, out, stream)
