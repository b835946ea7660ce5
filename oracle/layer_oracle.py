"""The definitions of what stands around a decoder layer's products, in numpy: norm and gated activation with INT8 outputs, tokens sorted by
expert and back.

Test infrastructure only; written from the formulas in include/liquidgemm.h.
"""
from __future__ import annotations

import numpy as np

from .attention_oracle import round_to


def quantise_rows(y):
    """y [M, K] float32 -> codes int8, scales float32: every operation one FP32 rounding."""
    scales = (np.abs(y).max(-1) / np.float32(127)).astype(np.float32)
    scales[scales == 0] = 1
    return np.clip(np.rint(y / scales[:, None]), -127, 127).astype(np.int8), scales


def norm_quantise(x, residual, weight, eps, dtype):
    """Codes, scales, h and y (unrounded, float32) of rows x, residual (values of `dtype`, as float32); residual and weight may be None."""
    h = x if residual is None else round_to(x.astype(np.float32) + residual.astype(np.float32), dtype)
    mean = (h.astype(np.float64) ** 2).mean(-1)
    r = (1.0 / np.sqrt(mean + np.float64(np.float32(eps)))).astype(np.float32)
    y = h if weight is None else h * weight.astype(np.float32)
    y = (y * r[:, None]).astype(np.float32)
    return *quantise_rows(y), h, y


def gated(x):
    """silu(gate) * up of rows [gate | up], FP64."""
    gate, up = np.split(x.astype(np.float64), 2, -1)
    with np.errstate(over="ignore"):
        return gate / (1.0 + np.exp(-gate)) * up


def dispatch(experts, n_experts):
    """row_offsets [n_experts + 1], places [tokens, each], and each row's token, by a stable sort of the pairs."""
    ids = np.asarray(experts).reshape(-1)
    here = np.flatnonzero((ids >= 0) & (ids < n_experts))
    order = here[np.argsort(ids[here], kind="stable")]
    places = np.full(ids.shape, -1, dtype=np.int32)
    places[order] = np.arange(len(order), dtype=np.int32)
    offsets = np.concatenate(([0], np.cumsum(np.bincount(ids[here], minlength=n_experts)))).astype(np.int32)
    return offsets, places.reshape(np.shape(experts)), order // np.shape(experts)[1]


def combine(Y, places, weights):
    """The sum of each token's rows and of their absolute values, FP64."""
    there = (places >= 0) & (places < len(Y))
    w = np.where(there, 1.0 if weights is None else weights.astype(np.float64), 0.0)[..., None]
    x = np.zeros((*places.shape, Y.shape[1]))
    x[there] = Y.astype(np.float64)[places[there]]
    return (x * w).sum(1), np.abs(x * w).sum(1)


def combine_backward(grad, Y, places, weights, dtype):
    """grad_Y (rounded to `dtype` after an FP32 product; NaN where no place names the row), grad_weights and the sums of its terms' absolute
    values, FP64."""
    of_rows = np.full(Y.shape, np.nan, dtype=np.float32)
    of_weights, size = np.zeros((2, *places.shape))
    for t, row in enumerate(places):
        for j, p in enumerate(row):
            if 0 <= p < len(Y):
                of_rows[p] = round_to(grad[t].astype(np.float32) * np.float32(weights[t, j]), dtype)
                terms = grad[t].astype(np.float64) * Y[p].astype(np.float64)
                of_weights[t, j], size[t, j] = terms.sum(), np.abs(terms).sum()
    return of_rows, of_weights, size
