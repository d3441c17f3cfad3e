"""A batch of sequences over a pool of cache pages, as the tests of its operators need it."""
import numpy as np
import torch

from oracle import serving as sv
from paper_2502_12574_amd import binding as hb

DEV = "cuda:0"


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


class Batch:
    """Sequences with `past` cached rows and `new` new ones each, pages in no order; rows that nobody owns hold NaN."""

    def __init__(self, past, new, kv_heads=2, group=4, page=16, bits=16, seed=0, pad=0, spare=2, width=None, dtype=torch.bfloat16):
        g = torch.Generator().manual_seed(seed)
        self.past, self.new, self.H, self.G, self.page, self.bits = list(past), list(new), kv_heads, group, page, bits
        S, self.starts = len(past), np.concatenate([[0], np.cumsum(new)]).tolist()
        self.T = self.starts[-1] + pad
        need = [-(-(max(p, 0) + n) // page) for p, n in zip(past, new)]
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.width = max(need + [1]) + 1 if width is None else width
        self.table = [[-1] * self.width for _ in range(S)]
        it = iter(order)
        for s in range(S):
            mine = [next(it) for _ in range(need[s])]
            self.table[s][:len(mine)] = mine[:self.width]
        shape = (self.n_pages, kv_heads, 2, page, 128)
        rows = torch.randn(shape, generator=g).to(torch.bfloat16)
        owned = torch.zeros(self.n_pages, page, dtype=torch.bool)
        for s in range(S):
            for b, p in enumerate(self.table[s]):
                if p >= 0:
                    owned[p, :max(0, min(page, max(past[s], 0) + new[s] - b * page))] = True
        keep = owned[:, None, None, :, None]
        self.scales = None
        if bits == 8:
            top = rows.float().abs().amax(-1)
            scale = torch.where(keep[..., 0], top / 448, torch.full_like(top, float("nan")))
            code = (rows.float() / top[..., None] * 448).clamp(-448, 448).to(torch.float8_e4m3fn)
            code = torch.where(keep, code.view(torch.uint8), torch.full_like(code.view(torch.uint8), 0x7F))
            self.pages, self.scales = code.view(torch.float8_e4m3fn).to(DEV), scale.to(DEV)
        else:
            self.pages = torch.where(keep, rows, torch.full_like(rows, float("nan"))).to(DEV)
        self.gen, self.dtype = g, dtype

    def rows(self, heads, dtype=None):
        return torch.randn(heads, self.T, 128, generator=self.gen).to(dtype or self.dtype).to(DEV)

    def values(self):
        """the pool as float64, [page][head][K|V][row][128]"""
        if self.bits == 16:
            return f64(self.pages)
        return sv.e4m3(self.pages.view(torch.uint8).cpu().numpy()) * f64(self.scales)[..., None]

    def structs(self, max_rows=None):
        def i32(x):
            return torch.tensor(x, dtype=torch.int32, device=DEV)
        cache = hb.make_paged_cache(self.pages, self.scales, self.n_pages, self.H, self.page, self.bits)
        batch = hb.make_paged_batch(i32(self.table), i32(self.past), i32(self.starts), len(self.past), self.width, self.T,
                                    max(1, max(self.new)) if max_rows is None else max_rows)
        return cache, batch

    def workspace(self):
        return torch.zeros(hb.hi_paged_workspace_bytes(self.H * self.G, self.H), dtype=torch.uint8, device=DEV)


def attention_close(got, q, values, b, prescaled=0, what=""):
    """The kernels' errors against the definition, from their roundings: a weight to bf16 (half a step, 2^-8 of its part of the
    output), the output to bf16, and the fp32 scores (each of at most 160 roundings of 2^-24 of the sum of magnitudes, which a
    power of two turns into as much of a weight, in the weight and in the sum it is divided by)."""
    want, size, score = sv.paged_attention(f64(q), values, b.table, b.past, b.starts, b.page,
                                           np.log(2.0) if prescaled else None)
    got = f64(got)
    mine = ~np.isnan(want)
    assert np.isnan(got[~mine]).all(), f"rows of no sequence were written {what}"
    tol = 2.0 ** -8 * (size + np.abs(want)) * 1.01 + 2 * 160 * 2.0 ** -24 * score[..., None] * size + 2.0 ** -20 * size + 1e-30
    off = np.abs(got - want)[mine] / tol[mine]
    assert np.isfinite(got[mine]).all(), f"not finite {what}"
    assert off.size == 0 or off.max() <= 1, f"{off.max():.3g} times the bound {what}"
