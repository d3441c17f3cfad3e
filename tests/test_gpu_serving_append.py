"""hi_paged_append: rotary embedding by each sequence's positions, and rows into the pages, against the definitions."""
import numpy as np
import pytest
import torch

from oracle import projection as op
from oracle import serving as sv
from paper_2502_12574_amd import binding as hb
from serving_batch import DEV, Batch, f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def run(b, q, k, v, theta, scale, q_out=None, max_rows=None):
    q_out = torch.full(q.shape, float("nan"), dtype=BF, device=DEV) if q_out is None else q_out
    cache, batch = b.structs(max_rows)
    hb.hi_paged_append(torch.cuda.current_stream(), cache, batch, q, k, v, int(q.dtype == F32), q.shape[0], theta, scale, q_out)
    torch.cuda.synchronize()
    return q_out


def check(b, before, q, k, v, theta, scale, q_out):
    """Every row of the pool and every query row, written or not."""
    after, out = b.values(), f64(q_out)
    untouched = np.ones((b.n_pages, b.page), bool)
    seen = np.zeros(b.T, bool)
    for s, (past, n) in enumerate(zip(b.past, b.new)):
        if past < 0:
            continue
        at, pos = slice(b.starts[s], b.starts[s] + n), np.arange(past, past + n)
        seen[at] = True

        def turned(x):
            x = f64(x)[:, at]
            return (op.apply_rope(x, pos, theta) if theta else x), np.abs(x) + np.abs(np.roll(x, 64, -1))
        want, size = turned(q)
        # fp32 cosine, sine and products: three roundings of the pair's magnitudes; then the scale's and the one to bf16
        tol = scale * (np.abs(want) * 2.0 ** -8 + size * 2.0 ** -21)
        assert (np.abs(out[:, at] - want * scale) <= tol + 1e-37).all()
        (kk, ks), vv = turned(k), f64(v)[:, at]
        for i in range(n):
            blk = (past + i) // b.page
            page = b.table[s][blk] if blk < b.width else -1
            if not 0 <= page < b.n_pages:
                continue
            r = (past + i) % b.page
            untouched[page, r] = False
            for j, x, e in ((0, kk[:, i], ks[:, i] * 2.0 ** -21), (1, vv[:, i], 0.0)):
                got = after[page, :, j, r]
                if b.bits == 16:
                    tol = np.abs(x) * 2.0 ** -8 + e
                else:                                     # half a step of e4m3, at least half of the smallest one; the scale's roundings
                    unit = np.abs(x).max(-1, keepdims=True) / 448
                    tol = np.maximum(np.abs(x) * 2.0 ** -4, unit * 2.0 ** -10) * (1 + 2.0 ** -20) + 2 * e
                    codes = b.pages[page, :, j, r].view(torch.uint8).cpu().numpy()
                    top = (codes & 127).max(-1)
                    assert ((top == 0x7E) | (unit[:, 0] == 0)).all()       # the row's largest value has the largest code
                assert (np.abs(got - x) <= tol + 1e-37).all(), (s, i, j)
    assert np.isnan(out[:, ~seen]).all()
    same = (after == before) | (np.isnan(after) & np.isnan(before))
    assert same.transpose(0, 3, 1, 2, 4)[untouched].all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("past,new,kw", [
    ([0], [1], dict()), ([0, 5, 31], [1, 1, 1], dict(group=1, kv_heads=1)), ([15, 16, 17, 0], [3, 40, 0, 1], dict(page=16)),
    ([100, 7], [29, 90], dict(page=64, kv_heads=3, group=2, pad=5)), ([1000, 3], [1, 1100], dict(page=256, kv_heads=1, group=3)),
    ([3, -1, 20], [2, 4, 9], dict(page=32)), ([70], [700], dict(kv_heads=5, group=1)), ([9] * 70, [1] * 70, dict(kv_heads=1))])
def test_append(past, new, kw, bits, dtype):
    b = Batch(past, new, bits=bits, dtype=dtype, seed=len(past) + bits, **kw)
    q, k, v = b.rows(b.H * b.G), b.rows(b.H), b.rows(b.H)
    before = b.values()
    for theta, scale in ((500000.0, hb.HI_Q_PRESCALE), (0.0, 1.0)):
        check(b, before, q, k, v, theta, scale, run(b, q, k, v, theta, scale))


def test_append_far_positions():
    """The angles of a position past a million are formed in double precision."""
    b = Batch([0, 0], [3, 2], page=1024, kv_heads=1, group=2, spare=0, width=3000)
    b.past = [1 << 20, 3000001]
    for s in range(2):
        page, b.table[s][0] = b.table[s][0], -1
        b.table[s][b.past[s] // 1024] = page
    q, k, v = b.rows(2), b.rows(1), b.rows(1)
    before = b.values()
    check(b, before, q, k, v, 10000.0, 1.0, run(b, q, k, v, 10000.0, 1.0))


def test_append_positions_up_to_the_largest():
    """Past lengths that end near 2^31: the queries are turned, and the rows, beyond any table, go nowhere."""
    b = Batch([10, 5], [6, 2], page=16, kv_heads=1, group=2, width=2)
    b.past = [(1 << 31) - 3, (1 << 31) - 1]
    q, k, v = b.rows(2), b.rows(1), b.rows(1)
    before = b.values()
    check(b, before, q, k, v, 10000.0, 1.0, run(b, q, k, v, 10000.0, 1.0))


@pytest.mark.parametrize("bits", [16, 8])
def test_append_pages_that_are_not_there(bits):
    b = Batch([10, 30, 60], [30, 8, 12], page=16, bits=bits, seed=6, width=4)          # the last sequence runs past its table
    b.table[0][1], b.table[1][2] = -1, b.n_pages
    q, k, v = b.rows(8), b.rows(2), b.rows(2)
    before = b.values()
    check(b, before, q, k, v, 1e4, 1.0, run(b, q, k, v, 1e4, 1.0))


@pytest.mark.parametrize("starts,new", [([-3, 4, 99], [4, 8]), ([0, 6, 4], [6, 0]), ([3, 3, 1 << 30], [0, 9]), ([50, 60, 70], [0, 0])])
def test_append_row_starts_out_of_range(starts, new):
    b = Batch([0, 0], [12, 12], page=16)
    b.T = 12
    q, k, v = b.rows(8), b.rows(2), b.rows(2)
    b.starts = starts
    cache, batch = b.structs()
    out = torch.full(q.shape, float("nan"), dtype=BF, device=DEV)
    before = b.values()
    hb.hi_paged_append(torch.cuda.current_stream(), cache, batch, q, k, v, 0, 8, 0.0, 1.0, out)
    torch.cuda.synchronize()
    b.starts, b.new = [min(max(x, 0), 12) for x in starts], new
    check(b, before, q, k, v, 0.0, 1.0, out)


@pytest.mark.parametrize("bits", [16, 8])
def test_append_without_queries_and_in_place(bits):
    b = Batch([5, 40], [7, 2], bits=bits, seed=2)
    q, k, v = b.rows(8), b.rows(2), b.rows(2)
    cache, batch = b.structs()
    s = torch.cuda.current_stream()
    before = b.values()
    hb.hi_paged_append(s, cache, batch, None, k, v, 0, 0, 1e4, 1.0, None)
    mine = q.clone()
    hb.hi_paged_append(s, cache, batch, mine, k, v, 0, 8, 1e4, 0.5, mine)
    torch.cuda.synchronize()
    check(b, before, q, k, v, 1e4, 0.5, mine)


def test_8_bit_rows_of_zeros_small_values_and_values_that_are_not_numbers():
    b = Batch([0], [6], bits=8, kv_heads=1, group=1, page=16, dtype=F32)
    q, k, v = b.rows(1), b.rows(1), b.rows(1)
    v[0, 0] = 0
    v[0, 1] = 1e-35                                   # below 2^-100: stored as zeros
    v[0, 2] *= 1e30
    v[0, 3, 7] = float("nan")
    v[0, 4, 9] = float("inf")
    run(b, q, k, v, 0.0, 1.0)
    got, want = b.values()[b.table[0][0], 0, 1], f64(v)[0]
    assert (got[0] == 0).all() and (got[1] == 0).all()
    assert (np.abs(got[2] - want[2]) <= np.maximum(np.abs(want[2]) * 2.0 ** -4, np.abs(want[2]).max() / 448 * 2.0 ** -10) * 1.0001).all()
    rest = [i for i in range(128) if i != 7]
    assert np.isnan(got[3, 7]) and np.isfinite(got[3, rest]).all()
    assert np.isnan(got[4]).all() and np.isfinite(got[5]).all()


def test_append_replayed_with_other_lengths():
    b = Batch([0, 0, 0], [40, 40, 40], page=16, seed=11)
    b.new, b.T = [1, 1, 1], 3
    b.starts = [0, 1, 2, 3]
    q, k, v = b.rows(8), b.rows(2), b.rows(2)
    out = torch.empty_like(q)
    cache, batch = b.structs()
    past = batch._keepalive[1]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        hb.hi_paged_append(torch.cuda.current_stream(), cache, batch, q, k, v, 0, 8, 1e4, 1.0, out)
    for step in range(3):
        b.past = [3 + step, 15 + step, 39 - step]
        past.copy_(torch.tensor(b.past))
        k.copy_(torch.randn(k.shape, generator=b.gen))
        out.fill_(float("nan"))
        before = b.values()
        graph.replay()
        torch.cuda.synchronize()
        check(b, before, q, k, v, 1e4, 1.0, out)
