"""The operators of a served batch, as cases that can be timed and compared: what lies between the projections of a
layer when many sequences share one pool of cache pages.

A case is a dict of plain values; `op` says which operator a pass calls:

  norm    hi_add_rmsnorm   residual + x, its root-mean-square norm, the new residual
  w4      hi_linear_quantized  rows times a weight matrix of 4-bit codes with a scale and a zero for each 128 of a row
  append  hi_paged_append  rotary embedding of new rows at their sequences' positions; K and V enter the pages, in bf16
                           or as 8-bit rows (e4m3) with a scale each
  attn    hi_paged_attn    causal grouped-query attention of each sequence's new rows over its pages

Sizes are the repository's own (32 query / 8 KV heads of 128 channels, hidden size 4096, contexts up to half a million
rows) or generic: 1 to 64 sequences, pages of 16 to 256 rows, 1 to 8 query heads a KV head.  Inputs are N(0, 1) rows as
everywhere in the repository, some keys scaled up.

With `own` false, run() is the operators' plain form in elementary torch operations in 32 bits (angles in 64).
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128                                   # channels of a head
GROUP = 128                               # input channels of a 4-bit scale
THETA = 500000.0
EPS = 1e-5
PRESCALE = 0.12751743082459868            # log2(e) / sqrt(128)
DEV = "cuda:0"


def _norm(name, **kw):
    c = dict(name=name, op="norm", rows=1, d=4096, x_fp32=False, residual_fp32=False)
    c.update(kw)
    return c


def _w4(name, **kw):
    c = dict(name=name, op="w4", rows=1, n_in=4096, n_out=6144, x_heads=False, y_heads=False)
    c.update(kw)
    return c


def _paged(name, op, **kw):
    c = dict(name=name, op=op, seqs=1, past=1000, new=1, lens=1, kv_heads=8, group=4, page=64, bits=16)
    c.update(dict(in_fp32=False) if op == "append" else dict(prescaled=True))
    c.update(kw)
    return c


def listed():
    return [
        # one generated token of one sequence between two projections: a launch and its latency
        _norm("norm_token"),
        # a prompt's chunk of odd length with the residual stream kept in fp32: pure traffic
        _norm("norm_chunk", rows=8191, residual_fp32=True),
        # the Q/K/V projection of one token of one sequence: the read of the weights
        _w4("w4_token", y_heads=True),
        # the output projection of a batch of 29 sequences, heads side by side as the attention leaves them
        _w4("w4_batch", rows=29, n_in=8192, n_out=8192, x_heads=True),
        # a chunk's worth of rows, where the products and no longer the weights count
        _w4("w4_chunk", rows=1500, n_out=4096),
        # one token of each of 48 sequences entering an 8-bit cache
        _paged("append_tokens8", "append", seqs=48, past=9000, lens=3, bits=8, page=32),
        # prompts of two sequences entering a bf16 cache straight from the projection's fp32 accumulators
        _paged("append_prompts", "append", seqs=2, past=700, new=5000, lens=4, in_fp32=True),
        # one token of one short conversation: the chain of latencies
        _paged("decode_short", "attn"),
        # one token of each of 64 sequences of very different lengths, 8-bit pages: the read of the cache
        _paged("decode_ragged8", "attn", seqs=64, past=32000, lens=5, bits=8),
        # one token behind half a million rows: one sequence has to fill the chip
        _paged("decode_long", "attn", past=524288 - 77, page=256),
        # a chunk of a long prompt: the matrix cores
        _paged("chunk_prompt", "attn", past=28672 - 33, new=4001, page=128),
        # a chunk of a prompt in one batch with sequences that generate, 8-bit pages
        _paged("chunk_mixed8", "attn", seqs=16, past=8000, new=384, lens=6, bits=8, page=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Sizes over the ranges of the listed cases, odd ones among them; none costs more than the largest listed one."""
    op = rng.choice(["norm", "w4", "w4", "append", "attn", "attn", "attn"])
    if op == "norm":
        c = _norm("", d=8 * _log(rng, 64, 1024), rows=_log(rng, 1, 8191), x_fp32=rng.random() < 0.3,
                  residual_fp32=rng.random() < 0.5)
    elif op == "w4":
        n_in, n_out = GROUP * _log(rng, 4, 64), GROUP * _log(rng, 4, 64)
        rows = _log(rng, 1, 64) if rng.random() < 0.7 else _log(rng, 64, 1500)
        if rows > 64:
            n_in, n_out = min(n_in, 4096), min(n_out, 4096)
        c = _w4("", rows=rows, n_in=n_in, n_out=n_out, x_heads=rng.random() < 0.5, y_heads=rng.random() < 0.5)
    else:
        group = rng.choice([1, 2, 4, 4, 7, 8])
        kw = dict(lens=rng.randrange(1000), kv_heads=rng.choice([1, 2, 4, 8, 8]), group=group,
                  page=rng.choice([16, 32, 64, 128, 256]), bits=rng.choice([16, 8]))
        if op == "append":
            seqs = _log(rng, 1, 48)
            kw.update(seqs=seqs, past=_log(rng, 1, 9000), new=_log(rng, 1, 5000 // seqs), in_fp32=rng.random() < 0.4)
        else:
            kw.update(prescaled=rng.random() < 0.5)
            kind = rng.choice(["decode", "decode", "few", "chunk"])
            if kind == "chunk":
                seqs, new = _log(rng, 1, 16), _log(rng, 17, 1024)
                kw.update(seqs=seqs, new=new, past=_log(rng, 1, max(2, min(28000, 3000000 // (seqs * new * group)))))
            else:
                seqs = _log(rng, 1, 64)
                kw.update(seqs=seqs, new=1 if kind == "decode" else rng.randint(2, 8),
                          past=_log(rng, 1, min(500000, 800000 // seqs)))
        c = _paged("", op, **kw)
    del c["name"]
    return c


def _lens(c):
    """(past lengths, numbers of new rows) of the case's sequences: the first has the case's own, the others up to that."""
    r = random.Random(c["lens"])
    past = [c["past"]] + [_log(r, max(1, c["past"] / 32), c["past"]) for _ in range(c["seqs"] - 1)]
    few = c["new"] > 64 and c["seqs"] > 8                # one prompt among sequences that generate
    new = [c["new"]] + [1 if few else r.randint(max(1, c["new"] // 2), c["new"]) for _ in range(c["seqs"] - 1)]
    return past, new


# ------------------------------------------------------------------------------------------------------- inputs


def _e4m3_rows(x):
    """rows of 128 values as (e4m3 codes, fp32 scales): scale = max |x| / 448, as the append writes them"""
    s = x.abs().amax(-1).float() * (1.0 / 448.0)
    return (x / s.clamp_min(1e-30).to(x.dtype).unsqueeze(-1)).clamp(-448, 448).to(torch.float8_e4m3fn), s


def _pool(c, g):
    """A cache whose pages all hold rows, and a page table that has the sequences' pages in no order."""
    past, new = _lens(c)
    need = [-(-(p + n) // c["page"]) for p, n in zip(past, new)]
    n_pages, width = sum(need) + 3, max(need) + 1
    shape = (n_pages, c["kv_heads"], 2, c["page"], D)
    rows = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    rows[:, :, 0, ::13] *= 3                             # some keys that stand out
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    at = torch.tensor([sum(need[:i]) for i in range(len(need))], device=DEV)
    col = torch.arange(width, device=DEV)
    table = order[(at[:, None] + col).clamp_max(n_pages - 1)]
    table = torch.where(col < torch.tensor(need, device=DEV)[:, None], table, torch.full_like(table, -1)).contiguous()
    s = dict(table=table, past=torch.tensor(past, dtype=torch.int32, device=DEV),
             starts=torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=DEV),
             rows=sum(new), max_rows=max(new), max_len=max(p + n for p, n in zip(past, new)), pages=rows, scales=None)
    if c["bits"] == 8:
        s["pages"], s["scales"] = _e4m3_rows(rows)
    return s


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device=DEV).to(dtype)

    s = dict(case=c)
    if c["op"] == "norm":
        wide = torch.float32 if c["residual_fp32"] else torch.bfloat16
        s.update(x=normal(c["rows"], c["d"], dtype=torch.float32 if c["x_fp32"] else torch.bfloat16),
                 residual=2 * normal(c["rows"], c["d"], dtype=wide),
                 weight=(1 + 0.1 * torch.randn(c["d"], generator=g, device=DEV)).to(torch.bfloat16),
                 new_residual=torch.empty(c["rows"], c["d"], dtype=wide, device=DEV),
                 out=torch.empty(c["rows"], c["d"], dtype=torch.bfloat16, device=DEV))
    elif c["op"] == "w4":
        n_out, n_in = c["n_out"], c["n_in"]
        w = (torch.randn(n_out, n_in // GROUP, GROUP, generator=g, device=DEV) / math.sqrt(n_in)).to(torch.bfloat16).float()
        zero = w.amin(-1)
        scale = ((w.amax(-1) - zero) * (1.0 / 15.0)).to(torch.bfloat16)
        code = ((w - zero[..., None]) / scale.float()[..., None]).round().clamp(0, 15).to(torch.uint8).view(n_out, n_in)
        x = normal(c["rows"], n_in)
        if c["x_heads"]:
            x = x.view(c["rows"], n_in // D, D).transpose(0, 1).contiguous()
        y = (n_out // D, c["rows"], D) if c["y_heads"] else (c["rows"], n_out)
        s.update(x=x, codes=(code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), scale=scale.contiguous(),
                 zero=zero.to(torch.bfloat16).contiguous(), out=torch.empty(y, dtype=torch.bfloat16, device=DEV))
    else:
        s.update(_pool(c, g))
        heads, T = c["kv_heads"] * c["group"], s["rows"]
        if c["op"] == "append":
            dt = torch.float32 if c["in_fp32"] else torch.bfloat16
            s.update(q=normal(heads, T, D, dtype=dt), k=normal(c["kv_heads"], T, D, dtype=dt),
                     v=normal(c["kv_heads"], T, D, dtype=dt), q_out=torch.empty(heads, T, D, dtype=torch.bfloat16, device=DEV))
        else:
            q = torch.randn(heads, T, D, generator=g, device=DEV)
            s.update(q=(q * PRESCALE if c["prescaled"] else q).to(torch.bfloat16),
                     out=torch.empty(heads, T, D, dtype=torch.bfloat16, device=DEV))
    return s


# ------------------------------------------------------------------------------------------------------ a pass


def _handles(s):
    """The structs and the workspace that a program of the framework makes once for a cache and a batch."""
    if "cache" not in s:
        from paper_2502_12574_amd import binding as hb
        c = s["case"]
        s["cache"] = hb.make_paged_cache(s["pages"], s["scales"], s["pages"].shape[0], c["kv_heads"], c["page"], c["bits"])
        s["batch"] = hb.make_paged_batch(s["table"], s["past"], s["starts"], c["seqs"], s["table"].shape[1], s["rows"],
                                         s["max_rows"])
        if c["op"] == "attn":
            heads = c["kv_heads"] * c["group"]
            s["workspace"] = torch.zeros(hb.hi_paged_workspace_bytes(heads, c["kv_heads"]), dtype=torch.uint8, device=DEV)
    return s["cache"], s["batch"]


def _run_own(s):
    from paper_2502_12574_amd import binding as hb
    c, stream = s["case"], torch.cuda.current_stream()
    if c["op"] == "norm":
        hb.hi_add_rmsnorm(stream, s["x"], int(c["x_fp32"]), s["residual"], int(c["residual_fp32"]), s["weight"], c["rows"],
                          c["d"], EPS, s["new_residual"], s["out"])
        return s["out"], s["new_residual"]
    if c["op"] == "w4":
        hb.hi_linear_quantized(stream, s["x"], s["codes"], s["scale"], s["zero"], c["rows"], c["n_in"], c["n_out"],
                        int(c["x_heads"]), int(c["y_heads"]), s["out"])
        return s["out"]
    cache, batch = _handles(s)
    heads = c["kv_heads"] * c["group"]
    if c["op"] == "append":
        hb.hi_paged_append(stream, cache, batch, s["q"], s["k"], s["v"], int(c["in_fp32"]), heads, THETA, PRESCALE,
                           s["q_out"])
        return _appended(s)
    hb.hi_paged_attn(stream, cache, batch, s["q"], heads, int(c["prescaled"]), s["out"], s["workspace"])
    return s["out"]


def _appended(s):
    return (s["q_out"], s["pages"]) if s["scales"] is None else (s["q_out"], s["pages"], s["scales"])


def _row_places(s):
    """for each new row: its sequence, its number among the sequence's new rows, its position"""
    t = torch.arange(s["rows"], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(s["starts"], t, right=True) - 1
    off = t - s["starts"][seq]
    return seq, off.long(), (s["past"][seq] + off).long()


def _rotated(x, pos):
    w = torch.exp(torch.arange(D // 2, device=DEV, dtype=torch.float64) * (-math.log(THETA) / (D // 2)))
    angle = pos.double()[:, None] * w
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    a, b = x.float().chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _plain_append(s):
    seq, _, pos = _row_places(s)
    R = s["case"]["page"]
    page, row = s["table"][seq, pos // R].long(), pos % R
    s["q_out"].copy_(_rotated(s["q"], pos) * PRESCALE)
    k, v = _rotated(s["k"], pos), s["v"].float()
    kv = torch.stack([k, v], dim=1).permute(2, 0, 1, 3)                     # [row][head][K|V][128]
    if s["scales"] is None:
        s["pages"][page, :, :, row] = kv.to(torch.bfloat16)
    else:
        top = kv.abs().amax(-1)
        s["scales"][page, :, :, row] = top * (1.0 / 448.0)
        code = (kv * (448.0 / top).unsqueeze(-1)).clamp(-448, 448).to(torch.float8_e4m3fn)
        s["pages"].view(torch.uint8)[page, :, :, row] = code.view(torch.uint8)
    return _appended(s)


def _plain_attn(s):
    c = s["case"]
    S, H, G, R = c["seqs"], c["kv_heads"], c["group"], c["page"]
    seq, off, _ = _row_places(s)
    P = -(-s["max_len"] // R)
    pages = s["table"][:, :P].long().clamp_min(0)
    rows = s["pages"].view(torch.uint8)[pages].view(s["pages"].dtype)         # [S][P][H][K|V][R][128]
    L = P * R
    k = rows[:, :, :, 0].permute(0, 2, 1, 3, 4).reshape(S, H, L, D).float()
    v = rows[:, :, :, 1].permute(0, 2, 1, 3, 4).reshape(S, H, L, D).float()
    del rows
    if s["scales"] is not None:
        sc = s["scales"][pages].permute(0, 2, 3, 1, 4).reshape(S, H, 2, L, 1)
        k.mul_(sc[:, :, 0])
        v.mul_(sc[:, :, 1])
    N = s["max_rows"]
    at = (s["starts"][:-1, None].long() + torch.arange(N, device=DEV)).clamp_max(s["rows"] - 1)
    q = s["q"].float()[:, at].view(H, G, S, N, D).permute(2, 0, 1, 3, 4).reshape(S, H, G * N, D)
    w = torch.matmul(q * (math.log(2.0) if c["prescaled"] else 1.0 / math.sqrt(D)), k.transpose(2, 3)).view(S, H, G, N, L)
    sees = torch.arange(L, device=DEV) <= (s["past"][:, None] + torch.arange(N, device=DEV))[..., None]
    w.masked_fill_(~sees[:, None, None], float("-inf"))
    w.sub_(w.amax(-1, keepdim=True)).exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(S, H, G * N, L), v).view(S, H, G, N, D).div_(total)
    s["out"].copy_(o.permute(1, 2, 0, 3, 4).reshape(H * G, S, N, D)[:, seq, off])
    return s["out"]


def _plain_norm(s):
    h = s["x"].float() + s["residual"].float()
    s["new_residual"].copy_(h)
    s["out"].copy_(h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * s["weight"].float())
    return s["out"], s["new_residual"]


def _plain_w4(s):
    c = s["case"]
    n_out, n_in = c["n_out"], c["n_in"]
    code = torch.stack([s["codes"] & 15, s["codes"] >> 4], dim=-1).view(n_out, n_in // GROUP, GROUP)
    w = (code.float() * s["scale"].float()[..., None] + s["zero"].float()[..., None]).view(n_out, n_in)
    x = s["x"].transpose(0, 1).reshape(c["rows"], n_in) if c["x_heads"] else s["x"]
    y = torch.matmul(x.float(), w.t())
    s["out"].copy_(y.view(c["rows"], n_out // D, D).transpose(0, 1) if c["y_heads"] else y)
    return s["out"]


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "w4": _plain_w4, "append": _plain_append, "attn": _plain_attn}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    c = case
    if c["op"] == "norm":
        one = 2 + (4 if c["x_fp32"] else 2) + 2 * (4 if c["residual_fp32"] else 2)
        return {"bytes": c["rows"] * c["d"] * one + 2 * c["d"], "flops": 5 * c["rows"] * c["d"]}
    if c["op"] == "w4":
        weights = c["n_out"] * (c["n_in"] // 2 + 4 * (c["n_in"] // GROUP))
        return {"bytes": weights + 2 * c["rows"] * (c["n_in"] + c["n_out"]), "flops": 2 * c["rows"] * c["n_in"] * c["n_out"]}
    past, new = _lens(c)
    H, heads, T = c["kv_heads"], c["kv_heads"] * c["group"], sum(new)
    kv_row = H * 2 * (D * c["bits"] // 8 + (4 if c["bits"] == 8 else 0))
    if c["op"] == "append":
        wide = 4 if c["in_fp32"] else 2
        return {"bytes": T * (D * (wide * (heads + 2 * H) + 2 * heads) + kv_row), "flops": T * D * (4 * (heads + H) + 4 * H)}
    pairs = sum(n * p + n * (n + 1) // 2 for p, n in zip(past, new))
    return {"bytes": sum(p + n for p, n in zip(past, new)) * kv_row + 4 * T * heads * D, "flops": 4 * D * heads * pairs}


# ---------------------------------------------------------------------------------------- the definition in 64 bits


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "norm":
        h = s["x"].double() + s["residual"].double()
        size = torch.sqrt((h * h).sum(1) / c["d"] + EPS)
        return (h / size[:, None]) * s["weight"].double()[None, :], h
    if c["op"] == "w4":
        x = s["x"].double()
        if c["x_heads"]:
            x = torch.cat(list(x), dim=1)
        y = torch.zeros(c["rows"], c["n_out"], dtype=torch.float64, device=DEV)
        for j in range(c["n_in"] // GROUP):
            part = s["codes"][:, j * GROUP // 2:(j + 1) * GROUP // 2].to(torch.int64)
            xs, sc, ze = x[:, j * GROUP:(j + 1) * GROUP], s["scale"][:, j].double(), s["zero"][:, j].double()
            y += (xs[:, 0::2] @ (part % 16).double().t() + xs[:, 1::2] @ (part // 16).double().t()) * sc
            y += xs.sum(1, keepdim=True) * ze
        return torch.stack(list(y.split(D, dim=1))) if c["y_heads"] else y
    past, new = _lens(c)
    starts, table = s["starts"].tolist(), s["table"].tolist()
    H, G, R = c["kv_heads"], c["group"], c["page"]
    if c["op"] == "append":
        pages = s["pages"].double()
        scales = None if s["scales"] is None else s["scales"].double()
        q_out = torch.zeros(H * G, s["rows"], D, dtype=torch.float64, device=DEV)
        freq = torch.tensor([THETA ** (-2.0 * i / D) for i in range(D // 2)], dtype=torch.float64, device=DEV)
        for i in range(c["seqs"]):
            a, n = starts[i], new[i]
            turn = torch.polar(torch.ones(n, D // 2, dtype=torch.float64, device=DEV),
                               torch.arange(past[i], past[i] + n, device=DEV).double()[:, None] * freq[None, :])

            def turned(x):
                z = torch.complex(x[..., :D // 2], x[..., D // 2:]) * turn
                return torch.cat([z.real, z.imag], dim=-1)

            q_out[:, a:a + n] = turned(s["q"][:, a:a + n].double()) * PRESCALE
            k, v = turned(s["k"][:, a:a + n].double()), s["v"][:, a:a + n].double()
            for b in range(past[i] // R, (past[i] + n - 1) // R + 1):        # page by page
                lo, hi = max(b * R, past[i]), min((b + 1) * R, past[i] + n)
                for j, x in ((0, k), (1, v)):
                    part = x[:, lo - past[i]:hi - past[i]]
                    if scales is not None:
                        top = part.abs().amax(-1)
                        scales[table[i][b], :, j, lo - b * R:hi - b * R] = top / 448
                        part = part * (448 / top)[..., None]
                    pages[table[i][b], :, j, lo - b * R:hi - b * R] = part
        return (q_out, pages) if scales is None else (q_out, pages, scales)
    if sum(n * (p + n) for p, n in zip(past, new)) * H * G > 8e9:
        return None                                                         # (too long in 64 bits)
    out = torch.zeros(H * G, s["rows"], D, dtype=torch.float64, device=DEV)
    unit = math.log(2.0) if c["prescaled"] else 1.0 / math.sqrt(D)
    for i in range(c["seqs"]):
        p, n, a = past[i], new[i], starts[i]
        mine = torch.tensor(table[i][:-(-(p + n) // R)], device=DEV)
        hidden = torch.arange(p + n, device=DEV)[None, :] > torch.arange(p, p + n, device=DEV)[:, None]
        for h in range(H):
            x = s["pages"].view(torch.uint8)[mine, h].view(s["pages"].dtype).double()
            if s["scales"] is not None:
                x = x * s["scales"][mine, h].double()[..., None]
            k, v = x[:, 0].reshape(-1, D)[:p + n], x[:, 1].reshape(-1, D)[:p + n]
            for j in range(h * G, (h + 1) * G):
                w = torch.softmax((s["q"][j, a:a + n].double() @ k.t() * unit).masked_fill(hidden, -math.inf), dim=1)
                out[j, a:a + n] = w @ v
    return out
