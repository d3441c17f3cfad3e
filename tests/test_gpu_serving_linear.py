"""hi_weight_quantize and hi_linear_quantized against the definitions."""
import numpy as np
import pytest
import torch

from oracle import serving as sv
from paper_2502_12574_amd import binding as hb
from serving_batch import DEV, f64

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def weights(n_out, n_in, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (n_out, n_in // 2), generator=g, dtype=torch.uint8)
    scale = (torch.rand(n_out, n_in // 128, generator=g) * spread / 8 + 0.01).to(BF)
    zero = (torch.randn(n_out, n_in // 128, generator=g) * spread).to(BF)
    return codes.to(DEV), scale.to(DEV), zero.to(DEV)


def check(y, x, codes, scale, zero, what):
    s, z, c = f64(scale), f64(zero), sv.unpack_codes(codes.cpu().numpy()).astype(np.float64)
    w = sv.quantized_weight(codes.cpu().numpy(), s, z)
    want = f64(x) @ w.T
    # the sums' terms, 16 s (16 + c) / 16 and z - 16 s: a sum of 128 of them, then one of the groups, in fp32 (at most as many roundings in a row)
    s, z = np.repeat(s, 128, 1), np.repeat(z, 128, 1)
    size = np.abs(f64(x)) @ (np.abs(s) * (16 + c) + np.abs(z) + 16 * np.abs(s)).T
    tol = 2.0 ** -8 * np.abs(want) + (128 + s.shape[1] // 128 + 40) * 2.0 ** -24 * size + 1e-37
    off = np.abs(f64(y) - want) / tol
    assert np.isfinite(off).all() and off.max() <= 1, (what, float(off.max()))


def heads(x):
    return x.view(x.shape[0], -1, 128).transpose(0, 1).contiguous()


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 64, 65, 129, 200])
@pytest.mark.parametrize("n_in,n_out", [(128, 16), (256, 128), (640, 48), (1152, 384), (2048, 272)])
def test_linear(rows, n_in, n_out):
    codes, scale, zero = weights(n_out, n_in, rows + n_in)
    x = torch.randn(rows, n_in, generator=torch.Generator().manual_seed(rows)).to(BF).to(DEV)
    for xh in (0, 1):
        for yh in (0, 1):
            if yh and n_out % 128:
                continue
            y = torch.full((rows * n_out + 64,), float("nan"), dtype=BF, device=DEV)
            hb.hi_linear_quantized(torch.cuda.current_stream(), heads(x) if xh else x, codes, scale, zero, rows, n_in, n_out, xh, yh, y)
            torch.cuda.synchronize()
            assert torch.isnan(y[rows * n_out:]).all()
            got = y[:rows * n_out]
            got = got.view(n_out // 128, rows, 128).transpose(0, 1).reshape(rows, n_out) if yh else got.view(rows, n_out)
            check(got, x, codes, scale, zero, (rows, n_in, n_out, xh, yh))


@pytest.mark.parametrize("rows,n_in,n_out", [(1, 4096, 6144), (5, 8192, 1024), (40, 4096, 4096), (300, 4096, 2048), (1100, 1024, 1168),
                                             (700, 4096, 4096), (1490, 2048, 1936)])
def test_linear_at_model_sizes(rows, n_in, n_out):
    codes, scale, zero = weights(n_out, n_in, 7)
    x = torch.randn(rows, n_in, generator=torch.Generator().manual_seed(rows)).to(BF).to(DEV)
    y = torch.empty(rows, n_out, dtype=BF, device=DEV)
    hb.hi_linear_quantized(torch.cuda.current_stream(), x, codes, scale, zero, rows, n_in, n_out, 0, 0, y)
    torch.cuda.synchronize()
    check(y, x, codes, scale, zero, (rows, n_in, n_out))


def test_weights_of_every_kind():
    """Zero scales (constant groups), negative scales, codes all alike, and rows of x that are zero."""
    codes, scale, zero = weights(128, 512, 3)
    codes[0], codes[1] = 0, 255
    scale[2], scale[3], zero[4] = 0, -scale[3], 0
    for rows in (3, 70):
        x = torch.randn(rows, 512, generator=torch.Generator().manual_seed(1)).to(BF).to(DEV)
        x[1] = 0
        y = torch.empty(rows, 128, dtype=BF, device=DEV)
        hb.hi_linear_quantized(torch.cuda.current_stream(), x, codes, scale, zero, rows, 512, 128, 0, 0, y)
        torch.cuda.synchronize()
        check(y, x, codes, scale, zero, rows)
        assert (y[1] == 0).all()


def test_a_bad_row_of_x_stays_in_its_row():
    codes, scale, zero = weights(256, 256, 5)
    for rows in (4, 100):
        x = torch.randn(rows, 256, generator=torch.Generator().manual_seed(2)).to(BF).to(DEV)
        bad = x.clone()
        bad[2, 9], bad[3, 200] = float("nan"), float("inf")
        y, z = (torch.empty(rows, 256, dtype=BF, device=DEV) for _ in range(2))
        hb.hi_linear_quantized(torch.cuda.current_stream(), x, codes, scale, zero, rows, 256, 256, 0, 0, y)
        hb.hi_linear_quantized(torch.cuda.current_stream(), bad, codes, scale, zero, rows, 256, 256, 0, 0, z)
        torch.cuda.synchronize()
        keep = [r for r in range(rows) if r not in (2, 3)]
        assert torch.equal(y[keep], z[keep]) and torch.isnan(z[2]).all() and not torch.isfinite(z[3]).any()


@pytest.mark.parametrize("n_out,n_in", [(16, 128), (37, 256), (128, 1152)])
def test_quantized_weights_are_the_encoding(n_out, n_in):
    g = torch.Generator().manual_seed(n_out)
    w = torch.randn(n_out, n_in, generator=g).to(BF)
    w[0, :128] = 0.5                                           # a constant group
    w[1, :128] *= 1e-38                                        # a range below 2^-120
    codes = torch.full((n_out * n_in // 2 + 16,), 77, dtype=torch.uint8, device=DEV)
    scale, zero = (torch.empty(n_out, n_in // 128, dtype=BF, device=DEV) for _ in range(2))
    hb.hi_weight_quantize(torch.cuda.current_stream(), w.to(DEV), n_out, n_in, codes, scale, zero)
    torch.cuda.synchronize()
    c, s, z = sv.encode_weight(w.float().numpy())
    assert (codes[:n_out * n_in // 2].cpu().numpy().reshape(n_out, -1) == c).all()
    assert (f64(scale) == s).all() and (f64(zero) == z).all()
    assert (codes[n_out * n_in // 2:] == 77).all()


def test_linear_replayed_with_new_rows():
    codes, scale, zero = weights(256, 512, 9)
    x, y = torch.zeros(6, 512, dtype=BF, device=DEV), torch.empty(6, 256, dtype=BF, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        hb.hi_linear_quantized(torch.cuda.current_stream(), x, codes, scale, zero, 6, 512, 256, 0, 0, y)
    for k in range(3):
        x.copy_(torch.randn(6, 512, generator=torch.Generator().manual_seed(k)))
        graph.replay()
        torch.cuda.synchronize()
        check(y, x, codes, scale, zero, k)


def test_linear_of_more_rows_than_a_grid_dimension():
    rows, n_in, n_out = 65535 * 16 + 40, 128, 16
    codes, scale, zero = weights(n_out, n_in, 3)
    x = torch.randn(rows, n_in, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(BF)
    y = torch.full((rows, n_out), float("nan"), dtype=BF, device=DEV)
    hb.hi_linear_quantized(torch.cuda.current_stream(), x, codes, scale, zero, rows, n_in, n_out, 0, 0, y)
    torch.cuda.synchronize()
    for at in (0, rows // 2, rows - 300):
        check(y[at:at + 300], x[at:at + 300], codes, scale, zero, at)
    assert torch.isfinite(y).all()
