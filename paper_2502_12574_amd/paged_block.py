"""A layer's step over many sequences that share one pool of cache pages: the batch-serving entry points in the order a server calls them.

  hidden states -> hi_add_rmsnorm -> Q/K/V projection (hi_qkv_rope without rotation, or hi_linear_quantized)
                -> hi_paged_append (rotary embedding, K and V into the pages) -> hi_paged_attn
                -> output projection (hi_out_proj or hi_linear_quantized) -> the next block's hi_add_rmsnorm

Only buffers, page numbers and call order live here; every step runs in the library.
"""
from __future__ import annotations

import torch

from . import binding as hb


def _check_buffer(what, t, dtypes, device):
    dtypes = dtypes if isinstance(dtypes, tuple) else (dtypes,)
    if t.dtype not in dtypes or t.device != device or not t.is_contiguous():
        raise RuntimeError(f"{what}: {t.dtype} of strides {t.stride()} on {t.device}; wanted are contiguous rows of {dtypes} on {device}")


class QuantizedWeight:
    """A weight matrix [n_out][n_in] in 4 bits (hi_weight_quantize): codes, and a scale and a zero for each 128 of a row.  Made on the
    current stream."""

    def __init__(self, w: torch.Tensor):
        _check_buffer("weight", w, torch.bfloat16, w.device)
        self.n_out, self.n_in = w.shape
        self.codes = torch.empty(self.n_out, self.n_in // 2, dtype=torch.uint8, device=w.device)
        self.scales, self.zeros = (torch.empty(self.n_out, self.n_in // 128, dtype=torch.bfloat16, device=w.device) for _ in range(2))
        with torch.cuda.device(w.device):
            hb.hi_weight_quantize(torch.cuda.current_stream(), w, self.n_out, self.n_in, self.codes, self.scales, self.zeros)

    @property
    def shape(self):
        return self.n_out, self.n_in


class PagePool:
    """Cache pages of all layers, and which sequence has which.  A page number stands for one page in every layer.

    open() gives a sequence a slot, step() the batch of the next step (with pages for its new rows), close() takes the slot's
    pages back.  kv_bits: 16 (bf16 rows) or 8 (e4m3 with a scale a row)."""

    def __init__(self, n_layers, n_kv_heads, n_pages, page_rows=64, kv_bits=16, max_seqs=64, max_context=1 << 17, device="cuda:0"):
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.n_pages, self.page_rows, self.n_kv_heads = n_pages, page_rows, n_kv_heads
        shape = (n_pages, n_kv_heads, 2, page_rows, 128)
        dt = torch.bfloat16 if kv_bits == 16 else torch.float8_e4m3fn
        self.pages = [torch.empty(shape, dtype=dt, device=self.device) for _ in range(n_layers)]
        self.scales = [torch.empty(shape[:-1], dtype=torch.float32, device=self.device) if kv_bits == 8 else None for _ in range(n_layers)]
        self.caches = [hb.make_paged_cache(p, s, n_pages, n_kv_heads, page_rows, kv_bits) for p, s in zip(self.pages, self.scales)]
        self.table_pages = -(-max_context // page_rows)
        self.free = list(range(n_pages - 1, -1, -1))
        self.idle = list(range(max_seqs - 1, -1, -1))
        self.owned = [[] for _ in range(max_seqs)]
        self.length = [0] * max_seqs

    def open(self) -> int:
        if not self.idle:
            raise RuntimeError("no slot is free: the pool was made for fewer sequences")
        slot = self.idle.pop()
        self.length[slot] = 0
        return slot

    def _open(self, slot) -> bool:
        return 0 <= slot < len(self.owned) and slot not in self.idle

    def close(self, slot: int):
        if not self._open(slot):
            raise RuntimeError(f"slot {slot} is not open")
        self.free += reversed(self.owned[slot])
        self.owned[slot] = []
        self.idle.append(slot)

    def step(self, slots, new_rows, n_rows=None) -> hb.hi_paged_batch:
        """The batch of a step that brings new_rows[i] rows of slots[i], and the pages for them; n_rows: rows of the step's buffers,
        if there are more than that.  The sequences count as that much longer from here on."""
        slots, new_rows = list(slots), list(new_rows)
        total = sum(new_rows)
        if len(set(slots)) != len(slots) or not all(map(self._open, slots)) or any(n < 0 for n in new_rows) or len(slots) != len(new_rows):
            raise RuntimeError("a step takes open slots, each once, and a number of rows for each")
        if n_rows is not None and n_rows < total:
            raise RuntimeError(f"{total} new rows in buffers of {n_rows}")
        need = [max(0, -(-(self.length[s] + n) // self.page_rows) - len(self.owned[s])) for s, n in zip(slots, new_rows)]
        if any(len(self.owned[s]) + m > self.table_pages for s, m in zip(slots, need)):
            raise RuntimeError("a sequence would outgrow max_context")
        if sum(need) > len(self.free):                       # before anything changes hands
            raise RuntimeError(f"{sum(need)} pages wanted, {len(self.free)} free")
        fresh = iter(reversed(self.free))
        past, starts, table = [self.length[s] for s in slots], [0], []
        for s, n, m in zip(slots, new_rows, need):
            starts.append(starts[-1] + n)
            table.append(self.owned[s] + [next(fresh) for _ in range(m)])
        width = max([len(t) for t in table] + [1])
        rows = [t + [-1] * (width - len(t)) for t in table]
        flat = torch.tensor(past + starts + [p for row in rows for p in row], dtype=torch.int32).to(self.device)     # (one copy)
        k = len(slots)
        del self.free[len(self.free) - sum(need):]
        for s, n, t in zip(slots, new_rows, table):
            self.owned[s] = t
            self.length[s] += n
        return hb.make_paged_batch(flat[2 * k + 1:], flat[:k], flat[k:2 * k + 1], k, width, total if n_rows is None else n_rows,
                                   max(new_rows + [1]))


class PagedBlock:
    """The attention block of one layer over a PagePool: pre-norm, projections, attention.

    norm_weight bf16 [d_model]; w_qkv [(Hq + 2 Hkv) * 128][d_model] and w_o [d_model][Hq * 128], each a bf16 tensor or a
    QuantizedWeight.  max_rows: the most rows of a step."""

    def __init__(self, pool: PagePool, layer: int, norm_weight, w_qkv, w_o, max_rows: int, rope_theta: float = 500000.0, eps: float = 1e-5,
                 stream=None):
        self.pool, self.layer, self.theta, self.eps, self.max_rows = pool, layer, rope_theta, eps, max_rows
        self.norm_weight, self.w_qkv, self.w_o = norm_weight, w_qkv, w_o
        self.D, self.Hkv = w_o.shape[0], pool.n_kv_heads
        self.Hq = w_o.shape[1] // 128
        assert w_qkv.shape == ((self.Hq + 2 * self.Hkv) * 128, self.D) and w_o.shape[1] == self.Hq * 128 and norm_weight.shape == (self.D,)
        dev, heads = pool.device, self.Hq + 2 * self.Hkv
        for what, w in (("norm weight", norm_weight), ("w_qkv", w_qkv), ("w_o", w_o)):
            if not isinstance(w, QuantizedWeight):
                _check_buffer(what, w, torch.bfloat16, dev)
        self.stream = stream or torch.cuda.current_stream(dev)
        # a bf16 projection hands over its fp32 sums, so that queries, keys and values are rounded once, behind the rotation
        self.fp32 = not isinstance(w_qkv, QuantizedWeight)
        torch.cuda.current_stream(dev).synchronize()         # (the pool and the weights, before another stream uses them)
        with torch.cuda.stream(self.stream):                 # the block's own buffers belong to its stream
            self.qkv = torch.empty(heads * max_rows * 128, dtype=torch.float32 if self.fp32 else torch.bfloat16, device=dev)
            self.q = torch.empty(self.Hq * max_rows * 128, dtype=torch.bfloat16, device=dev)
            self.attn = torch.empty(self.Hq * max_rows * 128, dtype=torch.bfloat16, device=dev)
            self.h = torch.empty(max_rows, self.D, dtype=torch.bfloat16, device=dev)
            self.workspace = torch.zeros(hb.hi_paged_workspace_bytes(self.Hq, self.Hkv), dtype=torch.uint8, device=dev)

    def forward(self, x: torch.Tensor, residual, batch: hb.hi_paged_batch, y: torch.Tensor):
        """x bf16 [n][d_model], n = batch.n_rows: what the block before put out; residual bf16 or fp32 [n][d_model], to which x is added
        in place, or None; y bf16 [n][d_model] receives the block's output.  Enqueues on the block's stream, which the caller orders
        behind whatever makes x and residual; the tensors, and the batch, may be let go of when this returns."""
        n, dev = batch.n_rows, self.pool.device
        for t in (x, y) if residual is None else (x, y, residual):
            if t.shape != (n, self.D) or n > self.max_rows:
                raise RuntimeError(f"rows of {tuple(t.shape)} for a batch of {n}: the block takes [n][{self.D}], at most {self.max_rows}")
            _check_buffer("rows", t, (torch.bfloat16, torch.float32) if t is residual else torch.bfloat16, dev)
        if n == 0:
            return y
        s, cache = self.stream, self.pool.caches[self.layer]
        if s != torch.cuda.current_stream(dev):              # (where their memory would be given out again)
            for t in (x, y, residual, *batch._keepalive):
                if isinstance(t, torch.Tensor):
                    t.record_stream(s)
        # a launch goes to a stream of the current device
        with torch.cuda.device(self.pool.device):
            hb.hi_add_rmsnorm(s, x, 0, residual, int(residual is not None and residual.dtype == torch.float32), self.norm_weight, n, self.D,
                              self.eps, residual, self.h)
            q, row = self.qkv.data_ptr(), n * 128 * self.qkv.element_size()
            k, v = q + self.Hq * row, q + (self.Hq + self.Hkv) * row
            if self.fp32:
                hb.hi_qkv_rope(s, self.h, self.w_qkv, self.D, self.Hq, self.Hkv, n, 0, 0.0, 1, q, k, v, None)
            else:
                w = self.w_qkv
                hb.hi_linear_quantized(s, self.h, w.codes, w.scales, w.zeros, n, w.n_in, w.n_out, 0, 1, q)
            hb.hi_paged_append(s, cache, batch, q, k, v, int(self.fp32), self.Hq, self.theta, hb.HI_Q_PRESCALE, self.q)
            hb.hi_paged_attn(s, cache, batch, self.q, self.Hq, 1, self.attn, self.workspace)
            if isinstance(self.w_o, QuantizedWeight):
                w = self.w_o
                hb.hi_linear_quantized(s, self.attn, w.codes, w.scales, w.zeros, n, w.n_in, w.n_out, 1, 0, y)
            else:
                hb.hi_out_proj(s, self.attn, self.w_o, self.Hq, self.D, n, 0, y)
        return y
