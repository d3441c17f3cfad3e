"""fp64 oracle of the operators that serve a batch of sequences from a pool of cache pages.

TEST INFRASTRUCTURE ONLY (see the package docstring).

What is computed, each from its plain definition with all inputs widened to float64:
  rmsnorm           h = x + r; h / sqrt(mean(h^2) + eps) * w
  quantized_weight  zero + code * scale, codes [n_out][n_in / 2] (low nibble first), a pair for each 128 input channels
  encode_weight     the encoding itself, in binary32 with one rounding per step (floating point decides the codes)
  e4m3              the value of an 8-bit code: 1 sign, 4 exponent (bias 7), 3 fraction bits, no infinities
  paged_rows        a sequence's rows of one head, gathered page by page (pages that are not there give None)
  paged_attention   softmax(q K^T / sqrt(d)) V row by row over the rows that are there; a row that sees none gives zeros
Pins (tests/test_oracle_serving.py): exactly rounded sums on tiny inputs; every e4m3 code against its bits taken apart
with fractions; a paged sequence against the pinned attention oracle on the same rows laid out in one piece.
"""
from __future__ import annotations

import numpy as np

WEIGHT_GROUP = 128


def rmsnorm(x, r, w, eps):
    h = np.asarray(x, np.float64) + (0.0 if r is None else np.asarray(r, np.float64))
    return h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64), h


def unpack_codes(codes):
    codes = np.asarray(codes, np.uint8)
    return np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)


def quantized_weight(codes, scales, zeros):
    c = unpack_codes(codes).astype(np.float64)
    n_out, n_in = c.shape
    c = c.reshape(n_out, n_in // WEIGHT_GROUP, WEIGHT_GROUP)
    return (c * np.asarray(scales, np.float64)[..., None] + np.asarray(zeros, np.float64)[..., None]).reshape(n_out, n_in)


def bf16_round(x):
    """float32 values rounded to bf16 (nearest, ties to even), as float32"""
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)


def encode_weight(w):
    """(codes, scales, zeros) of float32 weights that bf16 holds exactly"""
    w = np.asarray(w, np.float32)
    n_out, n_in = w.shape
    g = w.reshape(n_out, n_in // WEIGHT_GROUP, WEIGHT_GROUP)
    zero = g.min(-1)
    scale = bf16_round((g.max(-1) - zero) * (np.float32(1) / np.float32(15)))
    scale = np.where(scale >= np.float32(2.0 ** -120), scale, np.float32(0))
    inv = np.where(scale > 0, np.float32(1) / np.where(scale > 0, scale, np.float32(1)), np.float32(0))
    c = np.minimum(np.rint((g - zero[..., None]) * inv[..., None]), 15).astype(np.uint8).reshape(n_out, n_in)
    return c[:, 0::2] | (c[:, 1::2] << 4), scale, zero


def e4m3(codes):
    codes = np.asarray(codes, np.uint8).astype(np.int64)
    sign, exp, frac = 1.0 - 2.0 * (codes >> 7), (codes >> 3) & 15, codes & 7
    value = np.where(exp == 0, frac / 8.0 * 2.0 ** -6, (1 + frac / 8.0) * 2.0 ** (exp - 7.0))
    return np.where((codes & 127) == 127, np.nan, sign * value)


def paged_rows(pages, table_row, head, n, page_rows):
    """(K, V, there): the first n rows of a sequence; pages [p][h][2][r][d] float64"""
    i = np.arange(n)
    b = i // page_rows
    table_row = np.asarray(table_row, np.int64)
    page = np.where(b < len(table_row), table_row[np.minimum(b, len(table_row) - 1)], -1)
    there = (page >= 0) & (page < pages.shape[0])
    x = pages[np.where(there, page, 0), head, :, i % page_rows]
    x = np.where(there[:, None, None], x, 0.0)
    return x[:, 0], x[:, 1], there


def attend(q, k, v, sees, scale):
    """query rows [n][d] over keys, sees [n][keys]: (outputs, sums of weights times |v|, sizes of the largest score)"""
    none = ~sees.any(1)
    s = np.where(sees, q @ k.T * scale, -np.inf)
    w = np.exp(s - np.where(none, 0.0, s.max(1))[:, None])
    w /= np.where(none, 1.0, w.sum(1))[:, None]
    size = np.where(sees, np.abs(q) @ np.abs(k).T * scale, 0.0).max(1)
    return w @ v, w @ np.abs(v), size


def paged_attention(q, pages, table, past, starts, page_rows, scale=None):
    """q [Hq][T][d] -> (out, weighted |v|, score size), rows of no sequence NaN"""
    hq, T, d = q.shape
    group = hq // pages.shape[1]
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, size, score = np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.zeros((hq, T))
    for s in range(len(past)):
        first = min(max(int(starts[s]), 0), T)
        rows = min(max(int(starts[s + 1]), 0), T) - first
        if past[s] < 0 or rows <= 0:
            continue
        at = slice(first, first + rows)
        for h in range(pages.shape[1]):
            k, v, there = paged_rows(pages, table[s], h, int(past[s]) + rows, page_rows)
            sees = there[None] & (np.arange(len(there))[None] <= int(past[s]) + np.arange(rows)[:, None])
            for j in range(h * group, (h + 1) * group):
                out[j, at], size[j, at], score[j, at] = attend(q[j, at], k, v, sees, scale)
    return out, size, score
