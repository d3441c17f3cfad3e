"""hi_add_rmsnorm against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import serving as sv
from paper_2502_12574_amd import binding as hb
from serving_batch import DEV, f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def inputs(rows, d, xt, rt, seed=0):
    g = torch.Generator().manual_seed(seed)
    x, r = torch.randn(rows, d, generator=g).to(xt).to(DEV), (3 * torch.randn(rows, d, generator=g)).to(rt).to(DEV)
    return x, r, (1 + 0.2 * torch.randn(d, generator=g)).to(BF).to(DEV)


def check(out, res, x, r, w, eps):
    want, h = sv.rmsnorm(f64(x), None if r is None else f64(r), f64(w), eps)
    # one rounding to bf16, and fp32 sums of at most 64 roundings in a row, halved by the root
    tol = np.abs(want) * (2.0 ** -8 + 2.0 ** -17) + 1e-37
    assert (np.abs(f64(out) - want) <= tol).all()
    if res is not None:
        half = 2.0 ** -8 if res.dtype == BF else 2.0 ** -24
        assert (np.abs(f64(res) - h) <= np.abs(h) * (half + 2.0 ** -23)).all()


@pytest.mark.parametrize("xt", [BF, F32])
@pytest.mark.parametrize("rt", [BF, F32])
@pytest.mark.parametrize("rows,d", [(1, 8), (1, 4096), (3, 504), (5, 520), (7, 1000), (2, 2048), (3, 2056), (4, 5120), (1, 8200),
                                    (2, 12296), (3, 16384), (257, 512), (1000, 1032)])
def test_norm(rows, d, xt, rt):
    x, r, w = inputs(rows, d, xt, rt, rows + d)
    out = torch.full((rows + 1, d), float("nan"), dtype=BF, device=DEV)
    res = torch.full((rows + 1, d), float("nan"), dtype=rt, device=DEV)
    hb.hi_add_rmsnorm(torch.cuda.current_stream(), x, int(xt == F32), r, int(rt == F32), w, rows, d, 1e-5, res, out)
    torch.cuda.synchronize()
    check(out[:rows], res[:rows], x, r, w, 1e-5)
    assert torch.isnan(out[rows:]).all() and torch.isnan(res[rows:]).all()           # nothing behind the last row


def test_norm_without_residual_and_in_place():
    x, r, w = inputs(9, 1536, BF, BF, 4)
    s = torch.cuda.current_stream()
    out = torch.empty_like(x)
    hb.hi_add_rmsnorm(s, x, 0, None, 0, w, 9, 1536, 1e-6, None, out)
    torch.cuda.synchronize()
    check(out, None, x, None, w, 1e-6)
    x2, r2 = x.clone(), r.clone()
    hb.hi_add_rmsnorm(s, x2, 0, r2, 0, w, 9, 1536, 1e-6, r2, x2)                       # both buffers in place
    torch.cuda.synchronize()
    check(x2, r2, x, r, w, 1e-6)


def test_norm_of_zeros_of_large_rows_and_of_infinities():
    w = torch.ones(64, dtype=BF, device=DEV)
    x = torch.zeros(4, 64, dtype=F32, device=DEV)
    x[1] = 1e15
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    out = torch.empty(4, 64, dtype=BF, device=DEV)
    hb.hi_add_rmsnorm(torch.cuda.current_stream(), x, 1, None, 0, w, 4, 64, 1e-5, None, out)
    torch.cuda.synchronize()
    assert (out[0] == 0).all() and (out[1] == 1).all()
    assert torch.isnan(out[2, 5]) and (out[2, :5] == 0).all() and torch.isnan(out[3]).all()


def test_norm_on_another_stream_and_replayed():
    s = torch.cuda.Stream()
    x, r, w = inputs(33, 4096, BF, F32, 8)
    out, res = torch.empty_like(x), torch.empty_like(r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        hb.hi_add_rmsnorm(torch.cuda.current_stream(), x, 0, r, 1, w, 33, 4096, 1e-5, res, out)
    for k in range(3):
        x.copy_(inputs(33, 4096, BF, F32, 20 + k)[0])
        graph.replay()
        torch.cuda.synchronize()
        check(out, res, x, r, w, 1e-5)


def test_norm_of_more_rows_than_a_grid_dimension():
    rows = (1 << 26) + 5                          # 4 rows to a workgroup of 256 lanes
    x = torch.randn(rows, 8, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(BF)
    w = torch.ones(8, dtype=BF, device=DEV)
    out = torch.full_like(x, float("nan"))
    hb.hi_add_rmsnorm(torch.cuda.current_stream(), x, 0, None, 0, w, rows, 8, 1e-5, None, out)
    torch.cuda.synchronize()
    for at in (0, (1 << 24) - 50, (1 << 26) - 95):
        check(out[at:at + 100], None, x[at:at + 100], None, w, 1e-5)
    assert torch.isfinite(out).all()
