"""Pins of the oracle of the batch-serving operators."""
import math
from fractions import Fraction

import numpy as np

from oracle import attention as oa
from oracle import serving as sv


def test_norm_against_exactly_rounded_sums():
    rng = np.random.default_rng(1)
    x, r, w = rng.standard_normal((3, 24)), rng.standard_normal((3, 24)), rng.standard_normal(24)
    y, h = sv.rmsnorm(x, r, w, 1e-5)
    for i in range(3):
        row = [a + b for a, b in zip(x[i], r[i])]
        unit = math.sqrt(math.fsum(a * a for a in row) / 24 + 1e-5)
        assert np.allclose(h[i], row, rtol=0, atol=1e-15)
        assert np.allclose(y[i], [a / unit * b for a, b in zip(row, w)], rtol=1e-14, atol=0)


def test_every_e4m3_code():
    got = sv.e4m3(np.arange(256))
    for c in range(256):
        sign, exp, frac = -1 if c & 128 else 1, (c >> 3) & 15, c & 7
        if exp == 15 and frac == 7:
            assert math.isnan(got[c])
            continue
        want = Fraction(frac, 8) * Fraction(1, 64) if exp == 0 else (1 + Fraction(frac, 8)) * Fraction(2) ** (exp - 7)
        assert Fraction(got[c]) == sign * want
    assert np.nanmax(got) == 448.0


def test_weight_encoding_is_the_nearest_level_and_exact_on_a_grid():
    rng = np.random.default_rng(2)
    w = sv.bf16_round(rng.standard_normal((4, 256)).astype(np.float32))
    codes, scale, zero = sv.encode_weight(w)
    c, back = sv.unpack_codes(codes), sv.quantized_weight(codes, scale, zero)
    s, z = np.repeat(scale, 128, 1).astype(np.float64), np.repeat(zero, 128, 1).astype(np.float64)
    for level in range(16):
        assert (np.abs(w - back) <= np.abs(w - (z + level * s)) + 1e-6 * s).all()
    grid = (rng.integers(0, 16, (2, 128)) * 0.5 - 3.0).astype(np.float32)
    grid[:, 0], grid[:, 1] = -3.0, 4.5
    assert (sv.quantized_weight(*sv.encode_weight(grid)) == grid).all()
    codes, scale, zero = sv.encode_weight(np.full((1, 128), -0.25, np.float32))
    assert scale[0, 0] == 0 and (sv.quantized_weight(codes, scale, zero) == -0.25).all()
    assert sv.unpack_codes(np.array([[0x21, 0x43]], np.uint8)).tolist() == [[1, 2, 3, 4]]


def test_paged_attention_is_attention_over_the_rows_in_one_piece():
    rng = np.random.default_rng(3)
    pages = rng.standard_normal((5, 1, 2, 16, 128))
    table, past, starts = np.array([[4, 1, 3]]), [35], [0, 6]
    q = rng.standard_normal((2, 6, 128))
    k, v, there = sv.paged_rows(pages, table[0], 0, 41, 16)
    assert there.all() and (k[16:32] == pages[1, 0, 0]).all() and (v[32:] == pages[3, 0, 1, :9]).all()
    out, size, _ = sv.paged_attention(q, pages, table, past, starts, 16)
    for j in range(2):
        full = np.zeros((41, 128))
        full[35:] = q[j]
        want = oa.attn_layer(full[None], k[None], v[None])[0][35:]
        assert np.allclose(out[j], want, rtol=1e-12, atol=1e-13)
    assert (size >= np.abs(out) - 1e-12).all()


def test_paged_attention_without_rows():
    pages = np.ones((2, 1, 2, 16, 128))
    q = np.ones((1, 4, 128))
    out, _, _ = sv.paged_attention(q, pages, [[-1, 0], [7, 7]], [16, 3], [0, 2, 3], 16)
    assert (out[0, 0] == 1).all()                       # its own page is there, the one before is not
    assert (out[0, 2] == 0).all()                       # no page at all
    assert np.isnan(out[0, 3]).all()                    # belongs to nobody
