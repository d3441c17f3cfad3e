"""The page pool's bookkeeping."""
import pytest

from paper_2502_12574_amd.paged_block import PagePool


def rows(batch):
    table, past, starts = batch._keepalive
    return table.view(batch.n_seqs, batch.table_pages).tolist(), past.tolist(), starts.tolist()


def pool(**kw):
    a = dict(n_layers=2, n_kv_heads=1, n_pages=6, page_rows=16, max_seqs=3, max_context=64, device="cpu")
    a.update(kw)
    return PagePool(**a)


def test_steps_grow_sequences_page_by_page():
    p = pool()
    a, b = p.open(), p.open()
    s = p.step([a, b], [17, 3])
    table, past, starts = rows(s)
    assert past == [0, 0] and starts == [0, 17, 20] and (s.n_seqs, s.n_rows, s.max_rows, s.table_pages) == (2, 20, 17, 2)
    assert len(set(table[0])) == 2 and table[1][1] == -1 and len(p.free) == 3
    table, past, starts = rows(p.step([b, a], [13, 16], n_rows=40))
    assert past == [3, 17] and starts == [0, 13, 29] and len(p.free) == 2 and len(p.owned[a]) == 3
    everyone = p.owned[a] + p.owned[b] + p.free
    assert sorted(everyone) == list(range(6))
    p.close(a)
    assert len(p.free) == 5 and a in p.idle
    c = p.open()
    assert c == a and rows(p.step([c], [1]))[1] == [0]


def test_refusals_change_nothing():
    p = pool()
    a, b = p.open(), p.open()
    p.step([a], [40])
    before = ([list(x) for x in p.owned], list(p.free), list(p.length))
    for slots, new, kw in (([a, b], [20, 49], {}), ([a], [25], {}), ([a, a], [1, 1], {}), ([2], [1], {}), ([-1], [1], {}), ([3], [1], {}), ([b], [-1], {}), ([a, b], [1], {}),
                           ([b], [5], dict(n_rows=4))):
        with pytest.raises(RuntimeError):
            p.step(slots, new, **kw)
        assert before == ([list(x) for x in p.owned], list(p.free), list(p.length))
    p.open()
    with pytest.raises(RuntimeError):
        p.open()
    p.close(b)
    for slot in (b, -1, 3):
        with pytest.raises(RuntimeError):
            p.close(slot)


def test_a_step_that_cannot_be_copied_to_the_device_changes_nothing(monkeypatch):
    p = pool()
    a = p.open()
    p.step([a], [20])
    before = ([list(x) for x in p.owned], list(p.free), list(p.length))

    def fails(*args, **kw):
        raise MemoryError
    with monkeypatch.context() as m:
        m.setattr("paper_2502_12574_amd.paged_block.torch.tensor", fails)
        with pytest.raises(MemoryError):
            p.step([a], [20])
    assert before == ([list(x) for x in p.owned], list(p.free), list(p.length))
    assert rows(p.step([a], [20]))[1] == [20]
