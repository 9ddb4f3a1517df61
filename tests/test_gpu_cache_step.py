"""The step over a cache that may have been shortened (scores left behind, rotary positions of its own), runs of the cache's
operators together, under streams and graphs, and what they refuse."""
import ctypes

import numpy as np
import pytest

import dinfer_inputs as di
from harness import GpuRun, make_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import cache_ops
    return cache_ops


def tiny_run(dtype, n_seq, block, lo, hi, seed, layers=2, room=0):
    cfg = di.configs.scaled(di.model_preset("tiny"), dtype=dtype, n_layers=layers, logit_scale=1.0)
    cfg, w, inp = make_case(di.Workload("cache", cfg, n_seq, block, lo, hi, threshold=0.9, seed_index=seed))
    g = GpuRun(cfg, w, inp, max(n_seq * block, int(inp.prefix_len.sum())), int(inp.prefix_len.max()) + block + room)
    g.ctx.kv.zero_()
    g.prefill()
    g.torch.cuda.synchronize()
    return cfg, w, inp, g


def block_state(g):
    return [t.clone() for t in (g.tokens, g.mask, g.conf, g.argmax, g.n_committed, g.ctx.kv)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n_seq,block", [(1, 32), (3, 13), (5, 64)])
def test_scored_step_is_the_step(dtype, n_seq, block):
    """Positions equal to the prefix, scores on the side: the same bits as dinfer_step; every layer's scores are the block's
    attention weights (they sum to one per query and head, layer 0's are those of queries and keys worked out here)."""
    cfg, w, inp, g = tiny_run(dtype, n_seq, block, 20, 900, 150 + n_seq)
    torch = g.torch
    tok0, mask0 = g.tokens.clone(), g.mask.clone()
    g.step(0.05)
    want = block_state(g)
    g.tokens.copy_(tok0)
    g.mask.copy_(mask0)
    width = int(inp.prefix_len.max()) + block + 4
    score = torch.full((cfg.n_layers, n_seq, cfg.n_heads, width), 0.25, device=g.dev)
    out = torch.full_like(score, -1.0)
    g.ctx.step_scored(g.tokens, g.mask, g.prefix_len, g.page_table, 0.05, 0, g.conf, g.argmax, g.n_committed,
                      position=g.prefix_len.clone(), score_in=score, score_out=out, decay=0.5)
    torch.cuda.synchronize()
    for a, b in zip(want, block_state(g)):
        assert torch.equal(a, b)
    for s in range(n_seq):
        n = int(inp.prefix_len[s]) + block
        assert (out[:, s, :, n:] == -1).all()
        gathered = out[:, s, :, :n] - 0.125
        assert (gathered.sum(-1) - block).abs().max() <= block * 2.0 ** -14
    # layer 0 from the definition
    f32 = (lambda a: di.configs.bf16_to_f32(a) if a.dtype == np.uint16 else a)
    emb, wq = f32(w["emb"]).astype(np.float64), f32(w["layers"][0]["wq"]).astype(np.float64)
    hd, nh = cfg.head_dim, cfg.n_heads
    for s in range(n_seq):
        p = int(inp.prefix_len[s])
        x = emb[inp.block_tokens[s]]
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + cfg.rms_eps) * w["layers"][0]["attn_gain"]
        q = (x @ wq.T).reshape(block, nh, hd)
        ang = (p + np.arange(block))[:, None] * cfg.rope_theta ** (-2.0 * np.arange(hd // 2) / hd)
        cs, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
        q = np.concatenate([q[..., :hd // 2] * cs - q[..., hd // 2:] * sn, q[..., hd // 2:] * cs + q[..., :hd // 2] * sn], -1)
        k = g.read_kv(s, 0, 0, p + block)[0].astype(np.float64).reshape(-1, nh, hd)
        for h in range(nh):
            z = q[:, h] @ k[:, h].T / np.sqrt(hd)
            e = np.exp(z - z.max(-1, keepdims=True))
            ref = (e / e.sum(-1, keepdims=True)).sum(0)
            got = out[0, s, h, :p + block].cpu().numpy().astype(np.float64) - 0.125
            # queries are kept to 2^-16 (two bfloat16 planes) or float32: a score moves by at most that of sum |q k| scale
            bar = 2 * np.abs(q[:, h]).max() * np.abs(k[:, h]).max() * np.sqrt(hd) * (2.0 ** -14) + 2.0 ** -14
            assert np.abs(got - ref).max() <= bar * ref.max(), (s, h)
    g.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_generation_over_a_shortened_cache(m, dtype):
    """A block is scored, the cache loses positions, the next block runs on the rest.  Keeping everything changes no bit; with
    positions dropped, layer 0's new keys and values (which depend on tokens and rotary positions alone) are those of
    the unshortened run, and what is dropped is what scored least."""
    cfg, w, inp, g = tiny_run(dtype, 2, 32, 100, 300, 160, room=200)
    torch, ns, S = g.torch, 2, 32
    stride = g.page_table.shape[1] + 12
    order = torch.randperm(400, generator=torch.Generator().manual_seed(3)).to(torch.int32)
    # a context with pages to spare, holding the same rows
    big = GpuRun(cfg, w, di.configs.WorkloadInputs(inp.prefix_tokens, inp.block_tokens, inp.mask_bits, inp.prefix_len,
                                                   order[:2 * stride].reshape(2, stride).numpy().copy(), 400), g.ctx.max_tokens, 700,
                 weights_buffer=g.ctx.weights)
    big.ctx.kv.zero_()
    big.prefill()
    pos = big.prefix_len.clone()
    width = 600
    score = torch.zeros((cfg.n_layers, ns, cfg.n_heads, width), device=g.dev)
    tok0, mask0 = big.tokens.clone(), big.mask.clone()
    for i in range(2):              # two denoising steps leave their weights
        big.ctx.step_scored(big.tokens, big.mask, big.prefix_len, big.page_table, 0.02, 0, big.conf, big.argmax, big.n_committed,
                            position=pos, score_in=score, score_out=score, decay=0.9)
    big.ctx.refresh_block_scored(big.tokens, big.prefix_len, big.page_table, position=pos, score_in=score, score_out=score)
    torch.cuda.synchronize()
    assert big.prefix_len.tolist() == [int(p) + S for p in inp.prefix_len] == pos.tolist()
    length = big.prefix_len.clone()

    def run(keep, table):
        new_table = table.to(g.dev)
        kept = torch.empty((cfg.n_layers, ns, cfg.n_heads, keep), dtype=torch.int32, device=g.dev)
        new_len, out = torch.empty(ns, dtype=torch.int32, device=g.dev), torch.empty_like(score)
        big.ctx.kv_evict(0, cfg.n_layers, keep, 4, 32, score, length, big.page_table, new_table, kept, new_len, score_out=out)
        p = length.clone()          # the next block's positions go on from the full length
        big.tokens.copy_(tok0)
        big.mask.copy_(mask0)
        big.ctx.step_scored(big.tokens, big.mask, new_len, new_table, 0.02, 0, big.conf, big.argmax, big.n_committed, position=p,
                            score_in=out, score_out=out)
        torch.cuda.synchronize()
        n = int(new_len[0])
        rows = [t.clone() for t in big.ctx.kv_read(0, new_table[0], n, S)]
        return kept, out, [t.clone() for t in (big.tokens, big.mask, big.conf, big.argmax, big.n_committed)], rows

    big.tokens.copy_(tok0)
    big.mask.copy_(mask0)
    full = score.clone()
    big.ctx.step_scored(big.tokens, big.mask, length, big.page_table, 0.02, 0, big.conf, big.argmax, big.n_committed, score_in=full, score_out=full)
    torch.cuda.synchronize()
    plain = [t.clone() for t in (big.tokens, big.mask, big.conf, big.argmax, big.n_committed)]
    plain_rows = big.ctx.kv_read(0, big.page_table[0], int(length[0]), S)
    most = int(length.max())
    pages = -(-(most + S) // 16)
    spare = order[2 * stride:2 * stride + 2 * pages].reshape(2, pages)
    kept, out, state, rows = run(most, spare)
    for a, b in zip(state, plain):
        assert torch.equal(a, b)
    assert torch.equal(out, full) and all(torch.equal(a, b) for a, b in zip(rows, plain_rows))
    keep = 77
    kept, out, state, rows = run(keep, spare)
    assert all(torch.equal(a, b) for a, b in zip(rows, plain_rows))
    for l in range(cfg.n_layers):
        for s in range(ns):
            n = int(length[s])
            for h in range(cfg.n_heads):
                ids = kept[l, s, h].cpu()
                assert (ids[1:] > ids[:-1]).all() and ids[:4].tolist() == [0, 1, 2, 3] and ids[-32:].tolist() == list(range(n - 32, n))
                x = score[l, s, h, :n].cpu()
                gone = torch.ones(n, dtype=torch.bool)
                gone[ids.long()] = False
                assert x[gone].max() <= x[ids[4:-32].long()].min()
    big.close()
    g.close()


def layer_run(m, c, bufs, words):
    """One layer's use: append, attend, score, evict."""
    c.ctx.kv_append(0, c.lens, c.d_past, c.d_table, bufs["q"], bufs["k"], bufs["v"], bufs["q_out"], q_gain=bufs["gain"], k_gain=bufs["gain"],
                    rotary=bufs["rot"], rotary_table=bufs["tab"])
    c.ctx.attend(0, c.lens, c.d_past, c.d_table, bufs["q_out"], bufs["out"], visible=words, lse=bufs["lse"])
    c.ctx.kv_score(0, c.lens, c.d_past, c.d_table, bufs["q_out"], bufs["score"], visible=words, lse=bufs["lse"])
    c.ctx.kv_evict(0, 1, 100, 2, 10, bufs["score"][None], bufs["len"], c.d_table, bufs["new_table"], bufs["kept"], bufs["new_len"],
                   score_out=bufs["score_out"])


def layer_case(m, dtype="bf16", seed=50):
    import torch
    c = m.Cache(dtype, 4, 64, [9, 0, 32], [1100, 20, 77], seed=seed, spare=40)
    nq = 8
    b = dict(q=c.randn(c.T, nq * 64), k=c.randn(c.T, 256), v=c.randn(c.T, 256), gain=torch.ones(64, device=m.DEV) * 1.5)
    b["q_out"], b["out"] = torch.empty_like(b["q"]), torch.empty_like(b["q"])
    b["lse"], b["score"] = torch.zeros(c.T, nq, device=m.DEV), torch.zeros(3, 4, 1200, device=m.DEV)
    b["score_out"] = torch.zeros(1, 3, 4, 1200, device=m.DEV)
    b["len"] = (c.d_past + torch.tensor(c.lens, dtype=torch.int32, device=m.DEV)).contiguous()
    b["new_table"], b["new_len"] = c.free[:21].reshape(3, 7).contiguous().to(m.DEV), torch.zeros(3, dtype=torch.int32, device=m.DEV)
    b["kept"] = torch.zeros(1, 3, 4, 100, dtype=torch.int32, device=m.DEV)
    b["rot"] = m.binding.rotary(48, True, 10000.0, "yarn", 4.0, 512)
    b["tab"] = m.binding.rotary_table(b["rot"], 1200)
    return c, b, m.word_tensor(m.tree_words(c.g, c.lens))


OUTS = ["q_out", "out", "lse", "score", "score_out", "kept", "new_len"]


def test_operators_together_and_captured(m):
    import torch
    c, b, words = layer_case(m)
    pool0 = c.pool.clone()
    layer_run(m, c, b, words)
    torch.cuda.synchronize()
    m.check_attention(c, b["q_out"], 2, b["out"], b["lse"], m_words(words))
    eager = [b[n].clone() for n in OUTS] + [c.pool.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer_run(m, c, b, words)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer_run(m, c, b, words)
    q0 = b["q"].clone()
    for rep in range(4):
        b["q"].mul_(0.5)                      # eager work on other queries between the replays
        layer_run(m, c, b, words)
        torch.cuda.synchronize()
        assert not torch.equal(b["out"], eager[1])
        b["q"].copy_(q0)
        c.pool.copy_(pool0)
        for n in OUTS:
            b[n].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n, want in zip(OUTS, eager):
            assert torch.equal(b[n], want), (rep, n)
        assert torch.equal(c.pool, eager[-1]), rep
    c.close()


def m_words(words):
    return [int(w) & ((1 << 64) - 1) for w in words.cpu().tolist()]


def test_two_contexts_on_two_streams(m):
    """Contexts have workspaces of their own: calls on them may overlap."""
    import torch
    cases = [layer_case(m, seed=51), layer_case(m, seed=52)]
    want = []
    for c, b, words in cases:
        layer_run(m, c, b, words)
        torch.cuda.synchronize()
        want.append([b[n].clone() for n in OUTS])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for rep in range(5):
        for (c, b, words), st in zip(cases, streams):
            with torch.cuda.stream(st):
                layer_run(m, c, b, words)
    torch.cuda.synchronize()
    for (c, b, words), w in zip(cases, want):
        for n, x in zip(OUTS, w):
            assert torch.equal(b[n], x), n
        c.close()


def test_pages_beyond_32_bits(m):
    """The same rows in pages whose elements are numbered from 2^32 on (a pool of 8 GiB and more): the same outputs and pages."""
    import copy
    import torch
    c, b, words = layer_case(m)
    far, fb = copy.copy(c), dict(b)
    first = 2 ** 32 // (2 * 4 * 64 * 16)                  # elements of a page
    far.ctx = m.binding.Context(c.cfg, first + c.n_pages, c.ns, 64, c.max_pos)
    pool = far.ctx.kv.view(torch.bfloat16).view(first + c.n_pages, -1)[first:]
    pool.copy_(c.pool.view(c.n_pages, -1))
    low = far.ctx.kv.view(torch.bfloat16).view(first + c.n_pages, -1)[:c.n_pages]
    low.zero_()
    far.d_table = torch.where(c.d_table >= 0, c.d_table + first, c.d_table)
    fb["new_table"] = b["new_table"] + first
    for n in OUTS:
        fb[n] = torch.zeros_like(b[n])
    layer_run(m, c, b, words)
    layer_run(m, far, fb, words)
    torch.cuda.synchronize()
    for n in OUTS:
        assert torch.equal(b[n], fb[n]), n
    assert torch.equal(pool.view(torch.int16), c.pool.view(c.n_pages, -1).view(torch.int16)) and (low == 0).all()
    far.close()
    c.close()


def test_refusals(m):
    """Bad arguments are refused before anything is launched: every output keeps what it held."""
    import torch
    c, b, words = layer_case(m, "f32")
    E, ctx = m.binding.DinferError, c.ctx
    pool0 = c.pool.clone()
    append = dict(layer=0, lens=c.lens, d_past=c.d_past, d_page_table=c.d_table, d_q=b["q"], d_k=b["k"], d_v=b["v"], d_q_out=b["q_out"])
    attend = dict(layer=0, lens=c.lens, d_past=c.d_past, d_page_table=c.d_table, d_q=b["q"], d_out=b["out"])
    score = dict(layer=0, lens=c.lens, d_past=c.d_past, d_page_table=c.d_table, d_q=b["q"], d_score_out=b["score"])
    evict = dict(first_layer=0, n_layers=1, keep=100, n_sink=2, n_recent=10, d_score=b["score"][None], d_len=b["len"], d_page_table=c.d_table,
                 d_new_page_table=b["new_table"], d_kept=b["kept"], d_new_len=b["new_len"])

    def refused(fn, base, code, **kw):
        with pytest.raises(E) as e:
            fn(**{**base, **kw})
        assert e.value.code == code, e.value

    rot = m.binding.rotary
    for fn, base in ((ctx.kv_append, append), (ctx.attend, attend), (ctx.kv_score, score)):
        refused(fn, base, -1, layer=1)
        refused(fn, base, -1, layer=-1)
        refused(fn, base, -1, lens=[9, -1, 32])
        four = dict(d_past=torch.zeros(4, dtype=torch.int32, device=m.DEV), d_page_table=c.d_table[[0, 1, 2, 0]].contiguous())
        if fn == ctx.kv_score:
            four["d_score_out"] = torch.zeros(4, 4, 1200, device=m.DEV)
        refused(fn, base, -1, lens=[9, 0, 32, 0], **four)                                      # more sequences than the context takes
        long = torch.zeros(1200, 512, device=m.DEV)
        refused(fn, base, -3, lens=[9, 0, 1137], d_q=long, **({"d_q_out": long, "d_k": long[:, :256], "d_v": long[:, :256]} if fn == ctx.kv_append else
                                                             {"d_out": long} if fn == ctx.attend else {}))
        with pytest.raises(ValueError):
            fn(**{**base, "lens": [9, 0, 32, 0]})
        refused(fn, base, -1, d_q=torch.zeros(c.T, 6 * 64, device=m.DEV)[:, :5 * 64], **({"d_q_out": b["q"][:, :320]} if fn == ctx.kv_append else
                                                                                 {"d_out": b["q"][:, :320]} if fn == ctx.attend else {}))
        refused(fn, base, -1, d_q=torch.zeros(c.T * 512 + 1, device=m.DEV)[1:].view(c.T, 512))            # not 16-byte aligned
        for bad in (b["q"].half(), b["q"].cpu(), b["q"][:-1], b["q"].t(), b["q"][:, ::2]):           # type, device, rows, layout
            with pytest.raises(ValueError):
                fn(**{**base, "d_q": bad})
        with pytest.raises(ValueError):
            fn(**{**base, "d_past": c.d_past.long()})
        with pytest.raises(ValueError):
            fn(**{**base, "d_page_table": c.d_table.t()})
    many = torch.zeros(65, 512, device=m.DEV)
    refused(ctx.attend, attend, -1, lens=[65, 0, 0], d_q=many, d_out=many, visible=torch.zeros(65, dtype=torch.int64, device=m.DEV))
    for bad in (-1.0, float("nan"), float("inf")):
        refused(ctx.attend, attend, -1, scale=bad)
        refused(ctx.kv_score, score, -1, scale=bad)
        refused(ctx.kv_score, score, -1, decay=bad)
        refused(ctx.kv_append, append, -1, eps=bad, q_gain=b["gain"])
    refused(ctx.kv_append, append, -1, rotary=rot(48, False))                                              # no table
    for dim in (66, 47):                                                                                   # more than a head, odd
        refused(ctx.kv_append, append, -1, rotary=rot(dim, False), rotary_table=torch.zeros(2, 1200, dim // 2, device=m.DEV))
    for kw in (dict(keep=0), dict(n_sink=-1), dict(n_sink=60, n_recent=50), dict(n_layers=2), dict(first_layer=1), dict(d_new_page_table=c.d_table),
               dict(score_out=b["score"][None]), dict(d_new_len=b["len"]), dict(keep=100000)):
        layers, keep = kw.get("n_layers", 1), kw.get("keep", 100)
        if layers > 1 or keep != 100:                      # tensors that fit the refused number
            kw = dict(kw, d_score=b["score"][None].expand(layers, -1, -1, -1).contiguous(), d_kept=torch.zeros(layers, 3, 4, keep, dtype=torch.int32, device=m.DEV))
        refused(ctx.kv_evict, evict, -1, **kw)
    refused(ctx.kv_evict, evict, -3, keep=113, d_kept=torch.zeros(1, 3, 4, 113, dtype=torch.int32, device=m.DEV))      # seven new pages hold 112
    for fn, base, kw in ((ctx.kv_append, append, dict(q_gain=b["gain"].double())), (ctx.kv_append, append, dict(k_gain=b["gain"][:60])),
                         (ctx.kv_append, append, dict(positions=b["len"])), (ctx.kv_append, append, dict(rotary=rot(64), rotary_table=b["tab"])),
                         (ctx.attend, attend, dict(visible=words[:-1])), (ctx.attend, attend, dict(lse=b["lse"][:-1])),
                         (ctx.kv_score, score, dict(lse=b["lse"][:, :4])), (ctx.kv_score, score, dict(score_in=b["score"][:, :, :100])),
                         (ctx.kv_evict, evict, dict(d_kept=b["kept"][..., :99])), (ctx.kv_evict, evict, dict(d_len=b["len"][:2])),
                         (ctx.kv_evict, evict, dict(d_score=b["score"][None, :2]))):
        with pytest.raises(ValueError):
            fn(**{**base, **kw})
    torch.cuda.synchronize()
    assert torch.equal(c.pool, pool0) and all((b[n] == 0).all() for n in ("lse", "score", "score_out", "kept", "new_len"))
    # nothing to do is no error
    ctx.attend(0, [0, 0, 0], c.d_past, c.d_table, b["q"], b["out"])
    ctx.kv_score(0, [0, 0, 0], c.d_past, c.d_table, b["q"], b["score"])
    ctx.kv_append(0, [0, 0, 0], c.d_past, c.d_table, b["q"], b["k"], b["v"], b["q_out"])
    torch.cuda.synchronize()
    assert torch.equal(c.pool, pool0) and (b["score"] == 0).all()
    c.close()


def test_lengths_and_page_ids_that_leave_the_buffers(m):
    """Cached lengths beyond the page-table row are pulled back, page ids outside the pool are brought inside, lengths of
    eviction outside the score rows are cut: every access stays in the buffers."""
    import torch
    c, b, words = layer_case(m, "bf16")
    c.d_past.copy_(torch.tensor([10 ** 9, -5, 1180], dtype=torch.int32))
    layer_run(m, c, b, words)
    torch.cuda.synchronize()
    assert torch.isfinite(b["out"]).all()
    limit = c.d_table.shape[1] * 16
    # sequence 0's tokens sit at the end of its page-table row
    k, v = ctx_rows(c, 0, limit - 9, 9)
    assert torch.equal(v, b["v"][:9].float())
    b["len"].copy_(torch.tensor([-3, 10 ** 9, 0], dtype=torch.int32))
    layer_run(m, c, b, words)
    torch.cuda.synchronize()
    assert b["new_len"].tolist() == [0, 100, 0] and (b["kept"][0, 0] == -1).all()
    c.d_table.copy_(torch.where(torch.rand(c.d_table.shape, device=m.DEV) < 0.5, torch.full_like(c.d_table, 10 ** 8), torch.full_like(c.d_table, -9)))
    layer_run(m, c, b, words)
    torch.cuda.synchronize()
    c.close()


def ctx_rows(c, s, first, n):
    return c.ctx.kv_read(0, c.d_table[s], first, n)
