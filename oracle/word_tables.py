"""CPU oracle for the word-table operators: lookup, its gradient, microscaled four-bit numbers and their product, written
from their definitions in double.  Test infrastructure, not product code.  Nothing here imports the GPU package.

    embed       out_i = scale * table[t_i], zeros where t_i names no row
    embed_grad  G_w = scale * sum_{i: t_i = w} grad_i
    microscale  blocks of 32 elements: e = floor(log2 max|x|) - 2 (at least -127), elements the nearest of
                0, .5, 1, 1.5, 2, 3, 4, 6 times 2^e (ties to the even place in that list, above 6 to 6) with x's sign
"""
from __future__ import annotations

import math

import numpy as np

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK, GROUP = 32, 128


def embed(table, tokens, scale):
    table = np.asarray(table, np.float64)
    out = np.zeros((len(tokens), table.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < table.shape[0]:
            out[i] = scale * table[t]
    return out


def embed_grad(grad, tokens, rows, scale):
    """(the gradient, the sum of the magnitudes of its terms, the number of terms of each row)"""
    grad = np.asarray(grad, np.float64)
    out, size, terms = np.zeros((rows, grad.shape[1])), np.zeros((rows, grad.shape[1])), np.zeros(rows, np.int64)
    for i, t in enumerate(tokens):
        if 0 <= t < rows:
            out[t] += grad[i]
            size[t] += np.abs(grad[i])
            terms[t] += 1
    return scale * out, abs(scale) * size, terms


def _nearest(t):
    """Place in SIZES of the nearest to t >= 0, ties to the even place."""
    d = np.abs(SIZES - t)
    best = np.nonzero(d == d.min())[0]
    return int(best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1])


def quantize(x):
    """(codes [rows, 64 g], scales [rows, 4 g]) as bytes, g = ceil(width / 128)"""
    x = np.asarray(x, np.float64)
    rows, width = x.shape
    groups = -(-width // GROUP)
    half = np.zeros((rows, groups * GROUP), np.uint8)
    scales = np.zeros((rows, groups * 4), np.uint8)
    for i in range(rows):
        for lo in range(0, width, BLOCK):
            b = x[i, lo:lo + BLOCK]
            if not np.all(np.isfinite(b)):
                scales[i, lo // BLOCK] = 255
                continue
            top = float(np.abs(b).max())
            e = max(math.frexp(top)[1] - 1 - 2, -127) if top > 0 else -127
            scales[i, lo // BLOCK] = e + 127
            for j, v in enumerate(b):
                half[i, lo + j] = _nearest(min(abs(v) * 2.0 ** -e, 6.0)) | (8 if math.copysign(1.0, v) < 0 else 0)
    return half[:, 0::2] | (half[:, 1::2] << 4), scales


def numbers(codes, scales, width):
    """The numbers that codes and scales stand for [rows, width]."""
    half = np.stack((codes & 15, codes >> 4), axis=2).reshape(codes.shape[0], -1)
    value = np.where(half > 7, -1.0, 1.0) * SIZES[half & 7]
    power = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (value * np.repeat(power, BLOCK, axis=1))[:, :width]


def product(a, b, scale):
    """(scale * a b^T, the sums of the magnitudes of its terms) for two matrices of numbers"""
    return scale * (a @ b.T), abs(scale) * (np.abs(a) @ np.abs(b).T)
