"""CPU oracle for dropout of a word table's rows and for grouped four-bit integers, written from their definitions in double
(the generator in 64-bit integers).  Test infrastructure, not product code.  Nothing here imports the GPU package.

    kept            element (i, j) is kept where 32 bits r_ij < round((1 - p) 2^32); r_ij from Philox4x32-10 at its place
    dropout         scale / (1 - p) * x where kept, else 0
    embed_dropout_grad   G_w = scale / (1 - p) * sum over t_i = w of grad_i where kept
    group_quantize  per group of a row: b = the least number rounded down to bfloat16, s = bfloat16(binary32((largest - b) / 15)), the next
                    one towards zero where b + 15 s is beyond binary32,
                    q = nearest integer to (x - b) / s, ties to even, in 0 .. 15
    group_product   scale * sum_k a_ik (q_jk s + b)
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128
BF16_MAX = float(np.uint32(0x7F7F0000).view(np.float32))


def philox(counter, seed):
    """Philox4x32-10 of four arrays of 32-bit counters (uint64) under a 64-bit seed."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, np.uint64) for x in counter]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def bits(rows, width, seed, step, first=0):
    """The 32 random bits of every element of rows first .. first + rows - 1."""
    i, c = np.meshgrid(np.arange(first, first + rows, dtype=np.uint64), np.arange(-(-width // 8), dtype=np.uint64), indexing="ij")
    out = np.zeros((rows, c.shape[1] * 8), np.uint64)
    for second in (0, 1):
        word = (1 << 30) + (second << 27) + ((step >> 32) & 0xFFFFFF)
        x = philox((c, i, np.full_like(c, step & 0xFFFFFFFF), np.full_like(c, word)), seed)
        for e in range(8):
            half = (x[e // 2] >> np.uint64(16 * (e % 2))) & np.uint64(0xFFFF)
            out[:, e::8] |= half << np.uint64(0 if second else 16)
    return out[:, :width]


def kept(rows, width, p, seed, step, first=0):
    return bits(rows, width, seed, step, first) < np.uint64(int(np.rint((1.0 - p) * 2.0 ** 32)))


def dropout(x, p, seed, step, scale=1.0):
    x = np.asarray(x, np.float64)
    factor = scale / (1.0 - p) if p < 1 else 0.0
    with np.errstate(invalid="ignore"):
        return np.where(kept(*x.shape, p, seed, step), x * factor, 0.0)


def embed_dropout_grad(grad, tokens, rows, p, seed, step, scale=1.0):
    """(the gradient, the sum of the magnitudes of its terms, the number of tokens of each row)"""
    grad = np.asarray(grad, np.float64)
    mask = kept(*grad.shape, p, seed, step)
    factor = scale / (1.0 - p) if p < 1 else 0.0
    out, size, terms = np.zeros((rows, grad.shape[1])), np.zeros((rows, grad.shape[1])), np.zeros(rows, np.int64)
    for i, t in enumerate(tokens):
        if 0 <= t < rows:
            d = np.where(mask[i], grad[i], 0.0)
            out[t] += d
            size[t] += np.abs(d)
            terms[t] += 1
    return factor * out, abs(factor) * size, terms


def _bf16_down(x):
    """The largest bfloat16 number not above x, at least the least finite one."""
    f = np.float32(x)
    b = int(f.view(np.uint32))
    cut = b & 0xFFFF0000
    if b >> 31 and cut != b:
        cut += 0x10000
    return max(float(np.uint32(cut).view(np.float32)), -BF16_MAX) + 0.0


def _bf16_nearest(f):
    """A binary32 number to the nearest bfloat16, ties to even."""
    b = int(np.float32(f).view(np.uint32))
    b = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    return float(np.uint32(b).view(np.float32))


def group_quantize(x, group):
    """(codes q [rows, padded width], steps [rows, groups], bases [rows, groups]) with groups = padded width / group"""
    x = np.asarray(x, np.float64)
    rows, width = x.shape
    room = -(-width // BLOCK) * BLOCK
    q, step, base = np.zeros((rows, room), np.int64), np.zeros((rows, room // group)), np.zeros((rows, room // group))
    for i in range(rows):
        for g in range(-(-width // group)):
            v = x[i, g * group:(g + 1) * group]
            if not np.all(np.isfinite(v)):
                step[i, g] = base[i, g] = math.nan
                continue
            b = _bf16_down(v.min())
            s = _bf16_nearest(np.float32((v.max() - b) / 15.0))
            if abs(b + 15.0 * s) > float(np.finfo(np.float32).max):      # the next one towards zero
                s = float((np.float32(s).view(np.uint32) - np.uint32(0x10000)).view(np.float32))
            step[i, g], base[i, g] = s, b
            if s != 0:                                # (below 0 where all numbers are below the least finite bfloat16)
                q[i, g * group:g * group + len(v)] = np.clip(np.rint((v - b) / s), 0, 15).astype(np.int64)
    return q, step, base


def group_numbers(q, step, base, width):
    group = q.shape[1] // step.shape[1]
    return (q * np.repeat(step, group, axis=1) + np.repeat(base, group, axis=1))[:, :width]


def group_layout(q):
    """The bytes of codes: of 128 elements word 4 h + j has those from 32 j + 8 h on, element 2 t at half byte t, 2 t + 1 at 4 + t."""
    rows, room = q.shape
    out = np.zeros((rows, room // 2), np.uint8)
    for k in range(room):
        at = k % BLOCK
        j, h, e = at // 32, at % 32 // 8, at % 8
        half = e // 2 + 4 * (e % 2)
        byte = k // BLOCK * 64 + 4 * (4 * h + j) + half // 2
        out[:, byte] |= (q[:, k] << (4 * (half % 2))).astype(np.uint8)
    return out


def group_product(a, q, step, base, scale):
    """(scale a w^T, the magnitudes that bound its error: scale times the sum over groups of (15 |s| + |b|) sum |a|)"""
    a = np.asarray(a, np.float64)
    group = q.shape[1] // step.shape[1]
    w = group_numbers(q, step, base, a.shape[1])
    size = np.zeros((a.shape[0], q.shape[1]))
    size[:, :a.shape[1]] = np.abs(a)
    size = size.reshape(a.shape[0], -1, group).sum(axis=2)
    return scale * (a @ w.T), abs(scale) * (size @ (15.0 * np.abs(step) + np.abs(base)).T)
