"""The batch-serving operators together: norm, projections, append, attention and output projection of a layer over a page pool."""
import numpy as np
import pytest
import torch

from oracle import projection as op
from oracle import serving as sv
from paper_2502_12574_amd import binding as hb
from paper_2502_12574_amd import synth
from paper_2502_12574_amd.attention_block import AttentionBlock
from paper_2502_12574_amd.paged_block import PagedBlock, PagePool, QuantizedWeight
from paper_2502_12574_amd.session import Session
from serving_batch import DEV, f64

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
D, HQ, HKV, THETA = 512, 8, 2, 10000.0


def weights(seed):
    w = synth.draw_weight(seed, synth.TENSOR_WQKV, 0, (HQ + 2 * HKV) * 128, D, device=DEV)
    return w, synth.draw_weight(seed, synth.TENSOR_WO, 0, D, HQ * 128, device=DEV), synth.draw_hidden(seed, 0, 7, 1, D, device=DEV)[0]


def near(got, want, what, rel):
    got = f64(got)
    assert got.shape == want.shape and np.isfinite(got).all(), what
    err = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert err <= rel, (what, err)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("quantized", [False, True])
def test_steps_of_a_layer(bits, quantized):
    """Three steps of three sequences: prompts, single tokens, and a prompt among tokens.  Each stage against the definition on the
    bits that the stage before it put out; a bf16 rounding is 2^-9 of a value in the mean square at most, so a stage is off by
    at most two of them (attention: the weights' and the output's), 2^-8, and fp32 sums by far less."""
    w_qkv, w_o, norm = weights(40)
    pool = PagePool(1, HKV, 40, page_rows=16, kv_bits=bits, max_seqs=4, max_context=1024, device=DEV)
    if quantized:
        w_qkv, w_o = QuantizedWeight(w_qkv), QuantizedWeight(w_o)
        dense = [sv.quantized_weight(w.codes.cpu().numpy(), f64(w.scales), f64(w.zeros)) for w in (w_qkv, w_o)]
    else:
        dense = [f64(w_qkv), f64(w_o)]
    block = PagedBlock(pool, 0, norm, w_qkv, w_o, 200, THETA)
    slots = [pool.open() for _ in range(3)]
    g = torch.Generator().manual_seed(bits)
    for step, new in enumerate(([70, 0, 33], [1, 1, 1], [1, 100, 1])):
        past = [pool.length[s] for s in slots]
        n, pad = sum(new), step                                   # (padding rows behind the last sequence)
        batch = pool.step(slots, new, n_rows=n + pad)
        x, r = (torch.randn(n + pad, D, generator=g).to(BF).to(DEV) for _ in range(2))
        r = r.float() if step == 1 else r
        r0, y = r.clone(), torch.empty(n + pad, D, dtype=BF, device=DEV)
        block.forward(x, r, batch, y)
        torch.cuda.synchronize()
        T = n + pad
        want, h = sv.rmsnorm(f64(x), f64(r0), f64(norm), block.eps)
        near(block.h[:T], want, "norm", 2.0 ** -8)
        near(r, h, "residual", 2.0 ** -8)
        qkv = (f64(block.h[:T]) @ dense[0].T).reshape(T, HQ + 2 * HKV, 128).transpose(1, 0, 2)
        near(block.qkv[:(HQ + 2 * HKV) * T * 128].view(-1, T, 128), qkv, "projection", 2.0 ** -8)
        qkv = f64(block.qkv[:(HQ + 2 * HKV) * T * 128].view(-1, T, 128))
        q = block.q[:HQ * T * 128].view(HQ, T, 128)
        table, starts = batch._keepalive[0].view(3, -1).tolist(), batch._keepalive[2].tolist()
        values = f64(pool.pages[0]) if bits == 16 else sv.e4m3(pool.pages[0].view(torch.uint8).cpu().numpy()) * f64(pool.scales[0])[..., None]
        for i in range(3):
            at, pos = slice(starts[i], starts[i + 1]), np.arange(past[i], past[i] + new[i])
            if new[i] == 0:
                continue
            near(q[:, at], op.apply_rope(qkv[:HQ, at], pos, THETA) * hb.HI_Q_PRESCALE, "queries", 2.0 ** -8)
            for j in range(HKV):
                k, v, there = sv.paged_rows(values, table[i], j, past[i] + new[i], 16)
                assert there.all()
                rel = 2.0 ** -8 if bits == 16 else 2.0 ** -4
                near(torch.tensor(k[past[i]:]), op.apply_rope(qkv[HQ + j, at], pos, THETA), "keys", rel)
                near(torch.tensor(v[past[i]:]), qkv[HQ + HKV + j, at], "values", rel)
        want, _, _ = sv.paged_attention(f64(q), values, table, past, starts, 16, np.log(2.0))
        attn = block.attn[:HQ * T * 128].view(HQ, T, 128)
        near(attn[:, :n], want[:, :n], "attention", 2.0 ** -7)
        full = f64(attn).transpose(1, 0, 2).reshape(T, -1)
        near(y[:n], full[:n] @ dense[1].T, "output", 2.0 ** -8)


def test_one_sequence_agrees_with_the_single_sequence_block():
    """The same prompt and tokens through AttentionBlock (contiguous cache in HBM) and through PagedBlock (norm weight one and rows of unit
    size, so that the norm changes nothing but its rounding)."""
    w_qkv, w_o, _ = weights(41)
    n, steps = 150, 4
    x = synth.draw_hidden(41, 0, 0, n + steps, D, device=DEV).float()
    x = (x / x.square().mean(-1, keepdim=True).sqrt()).to(BF)
    outs = []
    with Session(1, HKV, HQ // HKV, 1024, 256, mode=hb.HI_MODE_RESIDENT, out_fp32=0, q_prescaled=True) as ss:
        block = AttentionBlock(ss, 0, w_qkv, w_o, THETA)
        ys, past = [], 0
        for rows in [n] + [1] * steps:
            y = torch.empty(rows, D, dtype=BF, device=DEV)
            block.forward(x[past:past + rows].contiguous(), past, y)
            past += rows
            ys.append(y)
        ss.sync()
        outs.append(torch.cat(ys))
    pool = PagePool(1, HKV, 20, page_rows=32, max_seqs=1, max_context=1024, device=DEV)
    paged = PagedBlock(pool, 0, torch.ones(D, dtype=BF, device=DEV), w_qkv, w_o, 256, THETA, eps=0.0)
    slot, ys, past = pool.open(), [], 0
    for rows in [n] + [1] * steps:
        y = torch.empty(rows, D, dtype=BF, device=DEV)
        paged.forward(x[past:past + rows].contiguous(), None, pool.step([slot], [rows]), y)
        past += rows
        ys.append(y)
    torch.cuda.synchronize()
    outs.append(torch.cat(ys))
    # the rows differ by roundings to bf16 of hidden states, queries, keys, values, weights and outputs: at most six of 2^-9 in the mean square
    near(outs[1], f64(outs[0]), "blocks", 6 * 2.0 ** -9)


def test_a_decode_step_captured_once_serves_later_tokens():
    """Lengths, starts and page numbers are read on the device: one captured step is replayed as the sequences grow."""
    w_qkv, w_o, norm = weights(42)
    pools = [PagePool(1, HKV, 30, page_rows=16, max_seqs=2, max_context=256, device=DEV) for _ in range(2)]
    blocks = [PagedBlock(p, 0, norm, w_qkv, w_o, 64, THETA) for p in pools]
    g = torch.Generator().manual_seed(3)
    prompt = torch.randn(40, D, generator=g).to(BF).to(DEV)
    for p, b in zip(pools, blocks):
        slots = [p.open(), p.open()]
        b.forward(prompt, None, p.step(slots, [25, 15]), torch.empty(40, D, dtype=BF, device=DEV))
    x, y = torch.zeros(2, D, dtype=BF, device=DEV), torch.empty(2, D, dtype=BF, device=DEV)
    table = torch.full((2, 16), -1, dtype=torch.int32, device=DEV)
    past, starts = torch.zeros(2, dtype=torch.int32, device=DEV), torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    batch = hb.make_paged_batch(table, past, starts, 2, 16, 2, 1)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        blocks[0].stream = torch.cuda.current_stream()
        blocks[0].forward(x, None, batch, y)
    for _ in range(30):
        token = torch.randn(2, D, generator=g).to(BF).to(DEV)
        step = pools[0].step([0, 1], [1, 1])
        table[:, :step.table_pages] = step._keepalive[0].view(2, -1)
        past.copy_(step._keepalive[1])
        x.copy_(token)
        graph.replay()
        want = torch.empty(2, D, dtype=BF, device=DEV)
        blocks[1].forward(token, None, pools[1].step([0, 1], [1, 1]), want)
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_block_refuses_rows_that_do_not_fit():
    w_qkv, w_o, norm = weights(43)
    pool = PagePool(1, HKV, 8, page_rows=16, max_seqs=1, max_context=64, device=DEV)
    block = PagedBlock(pool, 0, norm, w_qkv, w_o, 8, THETA)
    slot = pool.open()
    batch = pool.step([slot], [9])
    x = torch.zeros(9, D, dtype=BF, device=DEV)
    with pytest.raises(RuntimeError):
        block.forward(x, None, batch, x)
    with pytest.raises(RuntimeError):
        block.forward(x[:4], None, batch, x[:4])


def test_block_refuses_rows_of_other_layouts_and_takes_none():
    w_qkv, w_o, norm = weights(44)
    pool = PagePool(1, HKV, 8, page_rows=16, max_seqs=1, max_context=64, device=DEV)
    block = PagedBlock(pool, 0, norm, w_qkv, w_o, 8, THETA)
    slot = pool.open()
    batch = pool.step([slot], [4])
    x, wide = torch.zeros(4, D, dtype=BF, device=DEV), torch.zeros(4, 2 * D, dtype=BF, device=DEV)
    for args in ((wide[:, :D], None, x), (x, None, wide[:, :D]), (x, wide[:, :D], x), (x, x[:2], x), (x.float(), None, x),
                 (x, x.to(torch.float16), x), (x.cpu(), None, x), (x, None, x.float())):
        with pytest.raises(RuntimeError):
            block.forward(*args[:2], batch, args[2])
    with pytest.raises(RuntimeError):
        PagedBlock(pool, 0, norm, w_qkv.t().contiguous().t(), w_o, 8, THETA)
    with pytest.raises(RuntimeError):
        QuantizedWeight(w_o.float())
    none = x[:0]
    assert block.forward(none, None, pool.step([], []), none) is none


def test_a_block_on_a_stream_of_its_own_while_memory_is_given_out_again():
    """Batches and rows are let go of at once: what the current stream allocates and fills next must not be theirs while the block runs."""
    w_qkv, w_o, norm = weights(45)
    g = torch.Generator().manual_seed(5)
    rows = [torch.randn(n, D, generator=g).to(BF) for n in (300, 40, 40, 40)]
    outs = []
    for own in (False, True):
        pool = PagePool(1, HKV, 60, page_rows=16, max_seqs=1, max_context=960, device=DEV)
        stream = torch.cuda.Stream() if own else None
        block, slot, ys = PagedBlock(pool, 0, norm, w_qkv, w_o, 300, THETA, stream=stream), pool.open(), []
        for x in rows:
            x = x.to(DEV)
            y = torch.empty_like(x)
            torch.cuda.current_stream().synchronize()
            block.forward(x, None, pool.step([slot], [x.shape[0]]), y)
            if own:
                shape = x.shape
                del x
                for _ in range(4):
                    torch.full(shape, float("nan"), dtype=BF, device=DEV)
                    torch.full((512,), -1, dtype=torch.int32, device=DEV)
            ys.append(y)
        torch.cuda.synchronize()
        outs.append(torch.cat(ys))
    assert torch.equal(*outs)
