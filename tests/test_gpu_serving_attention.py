"""hi_paged_attn against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2502_12574_amd import binding as hb
from serving_batch import DEV, Batch, attention_close, f64

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def attend(b, q, prescaled=0, max_rows=None, ws=None, out=None):
    out = torch.full(q.shape, float("nan"), dtype=BF, device=DEV) if out is None else out
    ws = b.workspace() if ws is None else ws
    cache, batch = b.structs(max_rows)
    hb.hi_paged_attn(torch.cuda.current_stream(), cache, batch, q, q.shape[0], prescaled, out, ws)
    torch.cuda.synchronize()
    return out


BATCHES = [
    # one token: the first ever, around the edges of blocks and tiles, long ones; many sequences of very different lengths
    ([0], [1], dict()), ([15], [1], dict()), ([16], [1], dict(group=1)), ([63], [1], dict(page=32)), ([64, 0, 65], [1, 1, 1], dict(group=8)),
    ([1000], [1], dict(page=64, kv_heads=1)), ([5003], [1], dict(page=256)), ([3, 700, 0, 2100, 31, 32, 33], [1] * 7, dict(kv_heads=3)),
    ([int(10 * 1.09 ** i) for i in range(70)], [1] * 70, dict(kv_heads=1, group=2)), ([40] * 300, [1] * 300, dict(kv_heads=1, group=1)),
    # a few tokens a sequence
    ([100, 0, 17], [3, 4, 1], dict()), ([500, 31], [8, 7], dict(group=7, page=32)), ([90, 10], [2, 5], dict(group=16, kv_heads=1)),
    ([300] * 9, [2] * 9, dict(group=3, page=128)),
    # chunks, of odd lengths, behind nothing and behind much, in one batch with single tokens; groups that do not divide a block
    ([0], [64], dict()), ([0], [257], dict(group=1, page=64)), ([777], [130], dict(group=8, kv_heads=1)), ([100, 3000, 0], [90, 1, 33], dict(page=128)),
    ([50, 0], [70, 200], dict(group=5, kv_heads=1)), ([2000], [300], dict(group=7, kv_heads=1, page=32)), ([12, 300], [100, 60], dict(group=16, kv_heads=1)),
    ([4000], [520], dict(kv_heads=1, page=256)), ([64] * 5, [100, 1, 1, 40, 1], dict(group=2, pad=7)),
    # nothing to do for some of them
    ([5, 20, 9], [0, 2, 0], dict(pad=3)), ([5, -1, 9], [30, 25, 1], dict(pad=2)),
]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("i", range(len(BATCHES)))
def test_attention(i, bits):
    past, new, kw = BATCHES[i]
    b = Batch(past, new, bits=bits, seed=i, **kw)
    q = b.rows(b.H * b.G)
    values, ws = b.values(), b.workspace()
    for prescaled in (0, 1):
        qq = (q.float() * hb.HI_Q_PRESCALE).to(BF) if prescaled else q
        for hint in (None, 1, 1 << 20):                                  # every kernel takes every batch
            attention_close(attend(b, qq, prescaled, hint, ws), qq, values, b, prescaled, (prescaled, hint))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("hint", [1, 1 << 20])
def test_attention_over_pages_that_are_not_there(bits, hint):
    b = Batch([100, 40, 5, 200], [2, 30, 3, 1], page=16, bits=bits, seed=3, pad=2)
    b.table[0][3], b.table[0][0] = -1, b.n_pages + 5
    b.table[1][1] = b.table[1][3] = -7
    b.table[2][0] = 1 << 30                            # these query rows see no key at all
    b.table[3] = [-1] * b.width
    b.table[3][5] = 0                                  # (its rows are another sequence's: shared)
    q = b.rows(8)
    values = np.nan_to_num(b.values(), nan=3.0)
    if bits == 16:
        b.pages.copy_(torch.tensor(values))
    else:
        b.pages.copy_(torch.nan_to_num(b.pages.float(), nan=3.0).to(b.pages.dtype))
        b.scales.copy_(torch.nan_to_num(b.scales, nan=1.0))
        values = b.values()
    out = attend(b, q, max_rows=hint)
    attention_close(out, q, values, b)
    assert (out[:, b.starts[2]:b.starts[3]] == 0).all()


@pytest.mark.parametrize("hint", [1, 1 << 20])
def test_attention_past_the_end_of_the_table(hint):
    b = Batch([10, 60], [40, 9], page=16, seed=5, width=3)             # 48 rows of table; the second sequence's rows see 48 keys
    q = b.rows(8)
    attention_close(attend(b, q, max_rows=hint), q, b.values(), b)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("hint", [1, 1 << 20])
def test_attention_of_positions_up_to_the_largest(bits, hint):
    b = Batch([48], [3], page=16, bits=bits, seed=6, width=3)          # every row sees the whole table
    q = b.rows(8)
    want = attend(b, q, max_rows=hint)
    attention_close(want, q, b.values(), b)
    b.past = [(1 << 31) - 2]
    assert torch.equal(attend(b, q, max_rows=hint), want)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("hint", [1, 1 << 20])
def test_attention_of_peaked_and_of_equal_keys(bits, hint):
    b = Batch([900, 333], [1, 60], bits=bits, seed=8, kv_heads=1, group=4, page=64)
    if bits == 8:                                      # scores of up to a few hundred
        b.scales[:, :, 0] *= 6
    else:
        b.pages[:, :, 0] *= 6
    q = b.rows(4)
    attention_close(attend(b, q, max_rows=hint), q, b.values(), b, what="peaked")
    if bits == 8:
        b.pages.view(torch.uint8)[:, :, 0] = 0x40      # 2.0
        b.scales[:, :, 0] = 0.01
    else:
        b.pages[:, :, 0] = 0.5
    attention_close(attend(b, q, max_rows=hint), q, b.values(), b, what="equal")


@pytest.mark.parametrize("hint", [1, 1 << 20])
def test_infinite_and_nan_values_reach_only_rows_that_see_them(hint):
    """Rows of one sequence stay in it; what a later position holds does not reach an earlier call's rows."""
    b = Batch([50, 80], [1, 1], page=16, seed=9)
    q = b.rows(8)
    want = attend(b, q, max_rows=hint)
    page = b.table[1][2]
    b.pages[page, 0, 1, 3, 5] = float("nan")
    b.pages[page, 0, 0, 4, 6] = float("inf")
    got = attend(b, q, max_rows=hint)
    assert torch.equal(got[:, :1], want[:, :1]) and torch.equal(got[4:], want[4:])
    assert torch.isnan(got[:4, 1].float()).any()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("past,new,kw", [
    ([100, 0], [4, 2], dict(group=4)), ([30], [90], dict(group=1, kv_heads=1, page=32)), ([5, 64, 200], [200, 33, 1], dict(group=4)),
    ([3000], [70], dict(group=8, kv_heads=1, page=64)), ([17], [150], dict(group=3, page=128)), ([40], [5], dict(group=16, kv_heads=1)),
    ([8, 90], [60, 3], dict(group=11))])
def test_infinite_and_nan_rows_of_a_step_reach_only_later_rows(past, new, kw, bits):
    """Rows at the end of a sequence's new ones: an element of V, a row's scale, a row of K that is not finite."""
    b = Batch(past, new, bits=bits, seed=10, **kw)
    q = b.rows(b.H * b.G)
    values = b.values()
    clean = {hint: attend(b, q, max_rows=hint) for hint in (1, 1 << 20)}
    bad = torch.zeros(q.shape, dtype=torch.bool)

    def poison(s, back, head, which, channel=None, x=float("nan")):
        """the row `back` from the sequence's last one, seen by the last back + 1 query rows"""
        pos = past[s] + new[s] - 1 - back
        page, r = b.table[s][pos // b.page], pos % b.page
        if channel is not None and bits == 16:
            b.pages[page, head, which, r, channel] = x
        elif channel is not None:
            b.pages.view(torch.uint8)[page, head, which, r, channel] = 0xFF
        elif bits == 8:
            b.scales[page, head, which, r] = x
        else:
            b.pages[page, head, which, r] = x
        every = channel is None or which == 0
        at = slice(b.starts[s + 1] - 1 - back, b.starts[s + 1])
        bad[head * b.G:(head + 1) * b.G, at, slice(None) if every else channel] = True

    last = b.H - 1
    poison(0, 0, 0, 1, 7, float("inf"))
    poison(0, 1, 0, 1, 100, float("-inf"))
    poison(0, 2, 0, 1, 33)
    if new[0] > 40:
        poison(0, 25, 0, 1, 64, float("inf"))
    if len(new) > 1:
        poison(1, 0, last, 1, None, float("inf"))
        poison(1, 1, 0, 0, 5)
    bad = bad.to(DEV)
    for hint, want in clean.items():
        got = attend(b, q, max_rows=hint)
        assert not torch.isfinite(got[bad]).any(), hint
        attention_close(torch.where(bad, want, got), q, values, b, what=hint)


@pytest.mark.parametrize("hint", [1, 64])
def test_overlapping_sequences_leave_the_workspace_fit(hint):
    """Row starts that go back give rows to several sequences (their outputs are anyone's); the call after it is as ever."""
    b = Batch([300] * 299, [1] * 299, page=64, seed=14, kv_heads=1)
    q, ws = b.rows(4), b.workspace()
    cache, batch = b.structs(hint)
    starts = batch._keepalive[2]
    starts.copy_(torch.tensor([0, 299] * 150))
    hb.hi_paged_attn(torch.cuda.current_stream(), cache, batch, q, 4, 0, torch.empty_like(q), ws)
    first = attend(b, q, 0, hint, ws)
    attention_close(first, q, b.values(), b)
    assert torch.equal(attend(b, q, 0, hint), first)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("past,new,hint", [([20000, 100, 3000], [1, 1, 1], 1), ([9000, 50], [3, 90], 1 << 20), ([40000], [5], 1 << 20)])
def test_attention_gives_the_same_bits_again(bits, past, new, hint):
    b = Batch(past, new, bits=bits, seed=12, page=64)
    q, ws = b.rows(8), b.workspace()
    first = attend(b, q, 0, hint, ws)
    for _ in range(3):
        assert torch.equal(attend(b, q, 0, hint, ws), first)
    attention_close(first, q, b.values(), b)


@pytest.mark.parametrize("hint", [1, 64])
def test_attention_replayed_with_other_lengths(hint):
    b = Batch([400, 400, 400], [8, 8, 8], page=16, seed=13)
    values, all_rows = b.values(), b.rows(8)
    cache, batch = b.structs(hint)
    _, past, starts = batch._keepalive
    ws, out = b.workspace(), torch.empty_like(all_rows)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        hb.hi_paged_attn(torch.cuda.current_stream(), cache, batch, all_rows, 8, 0, out, ws)
    for p, n in (([400, 3, 77], [8, 8, 8]), ([0, 0, 0], [1, 1, 1]), ([399, 20, 200], [2, 5, 0]), ([1, 407, 64], [8, 1, 3])):
        b.past, b.new, b.starts = p, n, np.concatenate([[0], np.cumsum(n)]).tolist()
        past.copy_(torch.tensor(p))
        starts.copy_(torch.tensor(b.starts))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        attention_close(out, all_rows, values, b, what=(p, n))
        eager = attend(b, all_rows, 0, hint, ws)
        mine = ~torch.isnan(eager.float())
        assert torch.equal(out[mine], eager[mine])


def test_two_streams_with_workspaces_of_their_own():
    b = [Batch([6000 + i, 50], [1, 2], seed=20 + i, page=32) for i in range(2)]
    q, ws = [x.rows(8) for x in b], [x.workspace() for x in b]
    out = [torch.full(x.shape, float("nan"), dtype=BF, device=DEV) for x in q]
    streams = [torch.cuda.Stream() for _ in b]
    structs = [x.structs(1) for x in b]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            hb.hi_paged_attn(streams[i], *structs[i], q[i], 8, 0, out[i], ws[i])
    torch.cuda.synchronize()
    for i in range(2):
        attention_close(out[i], q[i], b[i].values(), b[i])


def test_a_pool_of_more_than_4_gib():
    """Byte offsets beyond 32 bits: the pages in use lie at both ends of the pool."""
    pages = torch.zeros(70000, 1, 2, 128, 128, dtype=BF, device=DEV)              # 4.6 GB
    b = Batch([300], [1], kv_heads=1, page=128, seed=30)
    far = [69999, 3, 68000]
    for i, p in enumerate(far):
        pages[p] = b.pages[b.table[0][i]]
    q = b.rows(4)
    near = attend(b, q)
    values = b.values()
    attention_close(near, q, values, b)
    small, b.pages, b.n_pages, b.table = b.pages, pages, 70000, [far + [-1] * (b.width - 3)]
    assert torch.equal(attend(b, q), near)
    assert torch.equal(attend(b, q, max_rows=64), attend_small(b, small, far, q))


def attend_small(b, small, far, q):
    at = {p: i for i, p in enumerate(far)}
    b.pages, b.n_pages, b.table = torch.stack([b.pages[p] for p in far]), 3, [[at.get(p, -1) for p in b.table[0]]]
    return attend(b, q, max_rows=64)
