"""The native marshalling of the batch-serving calls hands the library what ctypes hands it."""
import ctypes as C

import pytest
import torch

from paper_2502_12574_amd import binding as hb

NAMES = ("hi_add_rmsnorm", "hi_linear_quantized", "hi_paged_append", "hi_paged_attn")
OTHERS = ("hi_prefill_group", "hi_decode_group", "hi_decode_group_ragged", "hi_qkv_rope", "hi_out_proj")


class _Stream:
    cuda_stream = 0x7F0000001230


@pytest.fixture
def seen(monkeypatch):
    """The four functions replaced by ones that note their arguments (structures field by field)."""
    L, calls, keep = hb.lib(), [], []

    class Fake:
        pass

    fake = Fake()
    for name in OTHERS:
        setattr(fake, name, getattr(L, name))
    for name in NAMES:
        def note(*a, _name=name):
            calls.append((_name, [[getattr(x.contents, f[0]) for f in x.contents._fields_] if hasattr(x, "contents") else x for x in a]))
            return -5
        f = C.CFUNCTYPE(C.c_int32, *getattr(L, name).argtypes)(note)
        keep.append(f)
        setattr(fake, name, f)
    monkeypatch.setattr(hb, "_lib", fake)
    monkeypatch.setattr(hb, "_native", None)
    hb._load_native()
    yield calls
    monkeypatch.undo()
    hb._native = None
    hb._load_native()


T = torch.zeros(64, dtype=torch.bfloat16)
CACHE = hb.make_paged_cache(T, None, 5, 2, 32)
BATCH = hb.make_paged_batch(T, T, T, 3, 7, 11, 4)
ORDINARY = [
    lambda: hb.hi_add_rmsnorm(_Stream(), T, 0, T[8:], 1, T, 3, 64, 1e-5, None, 0x7F0000001000, check=False),
    lambda: hb.hi_linear_quantized(None, T, T, T[8:], T, 3, 256, 128, 1, 0, T, check=False),
    lambda: hb.hi_paged_append(_Stream(), CACHE, BATCH, None, T, T[8:], 1, 0, 5e5, 0.125, None, check=False),
    lambda: hb.hi_paged_attn(0x7F0000001000, CACHE, BATCH, T, 8, 1, T, T[8:], check=False),
    lambda: hb.hi_paged_append(None, hb.hi_paged_cache(1, 2, 3, 4, 5, 6), hb.hi_paged_batch.from_buffer_copy(BATCH), None, T, T, 1, 0, 5e5, 0.125, None, check=False),
]
UNUSUAL = [
    lambda: hb.hi_add_rmsnorm(_Stream(), T, 0, T, 1, T, 3, 64, 1, None, T, check=False),                    # an int for a float
    lambda: hb.hi_paged_attn(None, C.byref(CACHE), BATCH, T, 8, 1, T, T, check=False),                      # a structure by reference
]


@pytest.mark.parametrize("i", range(len(ORDINARY) + len(UNUSUAL)))
def test_native_and_ctypes_agree(seen, monkeypatch, i):
    if hb._native is hb._CtypesOnly:
        pytest.skip("the native marshalling was not built for this interpreter")
    call, native, returned = (ORDINARY + UNUSUAL)[i], hb._native, []

    class Noting:
        def __getattr__(self, name):
            def go(*args):
                returned.append(getattr(native, name)(*args))
                return returned[-1]
            return go

    monkeypatch.setattr(hb, "_native", Noting())
    assert call() == -5
    assert returned == ([-5] if i < len(ORDINARY) else [None])
    first = seen.pop()
    monkeypatch.setattr(hb, "_native", hb._CtypesOnly)
    assert call() == -5
    assert first == seen.pop() and not seen


def test_a_copied_structure_is_its_own(seen):
    """What a copy holds counts, not what it was copied from."""
    batch = hb.hi_paged_batch.from_buffer_copy(BATCH)
    batch.n_rows = 99
    hb.hi_paged_attn(None, CACHE, batch, T, 8, 1, T, T, check=False)
    assert seen.pop()[1][2][5] == 99


def test_structures_in_the_wrong_place_are_refused(seen):
    for cache, batch in ((BATCH, CACHE), (CACHE, CACHE), (CACHE, bytes(40)), (None, 3.0)):
        with pytest.raises(C.ArgumentError):
            hb.hi_paged_attn(None, cache, batch, T, 8, 1, T, T, check=False)
    assert not seen
