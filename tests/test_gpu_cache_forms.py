"""The paged cache's operators in their larger forms, the step's rotary positions and the refresh's scores, and settings of the rotation that
change its angles."""
import math

import numpy as np
import pytest

import dinfer_inputs as di
import test_gpu_cache_ops as ops
from harness import GpuRun, make_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import cache_ops
    return cache_ops


def test_append_of_more_tokens_than_one_attention_call_takes(m):
    """32768 tokens of 2048 query heads behind page-table rows of 32768 positions: the same queries and pages as sequence by sequence.
    (Attention numbers the meetings of rows and positions in 31 bits and refuses them.)"""
    import torch
    ns, n, heads, group = 32, 1024, 32, 64
    c = m.Cache("bf16", heads, 64, [n] * ns, [3 * s for s in range(ns)], seed=90, columns=2048)
    g = torch.Generator(device=m.DEV).manual_seed(90)
    q = torch.empty(c.T, heads * group * 64, dtype=torch.bfloat16, device=m.DEV).normal_(generator=g)
    kv = torch.empty(c.T, 2 * heads * 64, dtype=torch.bfloat16, device=m.DEV).normal_(generator=g)
    k, v = kv.split(heads * 64, 1)
    with pytest.raises(m.binding.DinferError) as e:
        c.ctx.attend(0, c.lens, c.d_past, c.d_table, q, q)
    assert e.value.code == -2
    pool0 = c.pool.clone()
    out = torch.empty_like(q)
    for s in range(ns):
        at = slice(s * n, (s + 1) * n)
        c.ctx.kv_append(0, [n], c.d_past[s:s + 1], c.d_table[s:s + 1], q[at], k[at], v[at], out[at])
    pool = c.pool.clone()
    c.pool.copy_(pool0)
    c.ctx.kv_append(0, c.lens, c.d_past, c.d_table, q, k, v, q)      # in place
    torch.cuda.synchronize()
    assert not torch.equal(pool, pool0) and torch.equal(c.pool, pool)
    for s in range(ns):
        assert torch.equal(q[s * n:(s + 1) * n], out[s * n:(s + 1) * n]), s
    c.close()


def angles(r, n, scaling, theta, factor, original, fast, slow, magnitude):
    """Cosines and sines of positions 0 .. n-1 in float64."""
    import torch
    j = torch.arange(r // 2, dtype=torch.float64)
    f = (theta * factor ** (r / (r - 2)) if scaling == "ntk" else theta) ** (-2 * j / r)
    size = 1.0
    if scaling == "linear":
        f = f / factor
    if scaling == "yarn":
        corner = [r * math.log(original / (b * 2 * math.pi)) / (2 * math.log(theta)) for b in (fast, slow)]
        lo, hi = max(0, math.floor(corner[0])), min(r - 1, math.ceil(corner[1]))
        ramp = ((j - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = f * (1 - ramp) + f / factor * ramp
        size = magnitude or (0.1 * math.log(factor) + 1 if factor > 1 else 1.0)
    a = torch.arange(n, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()]) * size


def check_table(m, r, n, scaling, theta, factor, original=0, fast=32.0, slow=1.0, magnitude=0.0, set_betas=True):
    """Within half a step of float32 and what double leaves of an angle of 32767 (a few steps of 2^-52)."""
    import torch
    rot = m.binding.rotary(r, False, theta, scaling, factor, original, fast if set_betas else 0.0, slow if set_betas else 0.0, magnitude)
    got = m.binding.rotary_table(rot, n).cpu().double()
    ref = angles(r, n, scaling, theta, factor, original, fast, slow, magnitude)
    assert got.shape == ref.shape
    d = (got - ref).abs()
    assert (d <= 2.0 ** -24 * ref.abs() + 1e-9).all(), float(d.max())


@pytest.mark.parametrize("scaling,factor", [("plain", 1.0), ("linear", 3.3), ("ntk", 1.7), ("yarn", 3.3)])
@pytest.mark.parametrize("theta", [10000.0, 12345.67])
def test_rotary_rules_that_float32_cannot_hold(m, scaling, factor, theta):
    check_table(m, 64, 32768, scaling, theta, factor, 2048)


@pytest.mark.parametrize("r", [20, 64, 128])
@pytest.mark.parametrize("original,fast,slow,magnitude", [(2048, 32.0, 1.0, 0.0), (4096, 16.0, 2.5, 0.0), (300, 4.0, 4.0, 1.3), (8192, 100.0, 0.25, 0.7)])
def test_ramped_frequencies(m, r, original, fast, slow, magnitude):
    """The ramp's corners from other numbers of turns than 32 and 1, and a magnitude of one's own."""
    check_table(m, r, 5000, "yarn", 10000.0, 4.0, original, fast, slow, magnitude)
    if (fast, slow) == (32.0, 1.0):
        check_table(m, r, 5000, "yarn", 10000.0, 4.0, original, fast, slow, magnitude, set_betas=False)


@pytest.mark.parametrize("factor", [1.0, 0.5, 1e-6])
def test_ramped_frequencies_that_do_not_stretch(m, factor):
    """A factor of at most one leaves cosines and sines their size."""
    check_table(m, 64, 300, "yarn", 10000.0, factor, 2048)


def test_largest_scale(m):
    """A scale whose product with log2(e) is no float32 number is refused; below it scores of zero stay zero."""
    import torch
    c = m.Cache("bf16", 2, 64, [3], [200], seed=91)
    q = torch.zeros(3, 128, dtype=torch.bfloat16, device=m.DEV)
    out, lse, score = torch.ones_like(q), torch.empty(3, 2, device=m.DEV), torch.zeros(1, 2, 203, device=m.DEV)
    for scale in (3e38, 1.8e38):
        with pytest.raises(m.binding.DinferError):
            c.ctx.attend(0, [3], c.d_past, c.d_table, q, out, scale=scale, lse=lse)
        with pytest.raises(m.binding.DinferError):
            c.ctx.kv_score(0, [3], c.d_past, c.d_table, q, score, scale=scale)
    torch.cuda.synchronize()
    assert (out == 1).all() and (score == 0).all()
    c.ctx.attend(0, [3], c.d_past, c.d_table, q, out, scale=1e38, lse=lse)
    c.ctx.kv_score(0, [3], c.d_past, c.d_table, q, score, scale=1e38)
    m.check_attention(c, q, 1, out, lse, scale=1e38)
    assert (score - 3 / 203).abs().max() <= 3 / 203 * 2.0 ** -18
    c.close()


def test_another_current_gpu_is_refused(m):
    """Every operator, the scored step and the scored refresh want the context's GPU to be the current one."""
    import torch
    if torch.cuda.device_count() < 2:
        pytest.skip("needs two GPUs")
    c = m.Cache("bf16", 4, 64, [9], [40], seed=92)
    q, out, score = c.randn(9, 256), c.randn(9, 256), torch.zeros(1, 4, 60, device=m.DEV)
    n, kept = torch.zeros(1, dtype=torch.int32, device=m.DEV), torch.zeros(1, 1, 4, 5, dtype=torch.int32, device=m.DEV)
    tok, mask = torch.zeros(1, 32, dtype=torch.int32, device=m.DEV), torch.zeros(1, dtype=torch.int64, device=m.DEV)
    conf = torch.zeros(1, 32, device=m.DEV)
    with torch.cuda.device(1):
        for call in (lambda: c.ctx.kv_append(0, [9], c.d_past, c.d_table, q, q, q, out), lambda: c.ctx.attend(0, [9], c.d_past, c.d_table, q, out),
                     lambda: c.ctx.kv_score(0, [9], c.d_past, c.d_table, q, score),
                     lambda: c.ctx.kv_evict(0, 1, 5, 0, 0, score[None], c.d_past, c.d_table, c.d_table.clone(), kept, n),
                     lambda: c.ctx.step_scored(tok, mask, c.d_past, c.d_table, 0.5, 0, conf, tok.clone(), n),
                     lambda: c.ctx.refresh_block_scored(tok, c.d_past, c.d_table)):
            with pytest.raises(m.binding.DinferError, match="current device"):
                call()
    c.close()


# ------------------------------------------------------------------------------------------------ larger forms

@pytest.mark.parametrize("dtype,heads,hd", [("bf16", 35, 128), ("bf16", 35, 64), ("f32", 34, 128), ("f32", 33, 64)])
@pytest.mark.parametrize("dim,interleaved,scaling,norm,custom", [(0, False, "plain", True, False), (2, True, "ntk", False, True),
                                                                 (20, False, "yarn", True, True), (20, True, "linear", False, False)])
def test_append_four_heads_per_workgroup(m, monkeypatch, dtype, heads, hd, dim, interleaved, scaling, norm, custom):
    """64 ragged sequences fill the chip with workgroups of four heads (8192 meetings of pages and heads, the last workgroup's heads not all
    there): norms, both layouts of pairs, rotations that end inside a lane's features and those that do not."""
    lens, past = [7 * s % 41 for s in range(64)], [13 * s % 211 for s in range(64)]
    assert sum((n + 14) // 16 + 1 if n else 0 for n in lens) * heads * 2 >= 8192
    monkeypatch.setattr(ops, "APPENDS", [(lens, past)])
    ops.test_append(m, dtype, heads, hd, 0, dim, interleaved, scaling, norm, 1, custom)


@pytest.mark.parametrize("dtype,heads,hd", ops.SHAPES)
@pytest.mark.parametrize("past,keep,sink,recent", [([4000, 1025, 3], 1024, 4, 64), ([2049, 1024, 2048], 2048, 0, 0), ([1500], 1, 0, 0),
                                                   ([4094, 0, 1026], 777, 700, 77)])
def test_evict_up_to_4096_positions(m, dtype, heads, hd, past, keep, sink, recent):
    """Sixteen scores per thread of four waves."""
    assert 1024 < max(past) + 2 <= 4096
    ops.test_evict(m, dtype, heads, hd, past, keep, sink, recent)


# ------------------------------------------------------------------------------------------------ the step

def run_of(dtype, n_seq, block, lo, hi, seed, columns):
    """The tiny model behind ragged prompts, page-table rows of `columns` pages."""
    cfg = di.configs.scaled(di.model_preset("tiny"), dtype=dtype, n_layers=2, logit_scale=1.0)
    cfg, w, inp = make_case(di.Workload("forms", cfg, n_seq, block, lo, hi, threshold=0.9, seed_index=seed))
    table = np.random.default_rng(seed).permutation(n_seq * columns).astype(np.int32).reshape(n_seq, columns)
    inp = di.configs.WorkloadInputs(inp.prefix_tokens, inp.block_tokens, inp.mask_bits, inp.prefix_len, table, n_seq * columns)
    g = GpuRun(cfg, w, inp, max(n_seq * block, int(inp.prefix_len.sum())), columns * 16)
    g.ctx.kv.zero_()
    g.prefill()
    return cfg, w, inp, g


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n_seq,block", [(1, 32), (2, 32), (3, 40), (5, 64), (16, 64)])
def test_positions_of_ones_own(dtype, n_seq, block):
    """The first layer's keys and values depend on tokens and rotary positions alone: those of a block behind p cached positions that is turned
    as at P are, bit for bit, those of the same block behind P cached positions.  (By the number of tokens all forms of the projection.)"""
    cfg, w, inp, g = run_of(dtype, n_seq, block, 20, 300, 170 + n_seq, 40)
    torch = g.torch
    tok0, mask0 = g.tokens.clone(), g.mask.clone()
    p = g.prefix_len.clone()
    at = (p + 40 * torch.arange(n_seq, device=g.dev, dtype=torch.int32) % 170 - 11).contiguous()

    def rows(first):
        return [torch.cat([g.ctx.kv_read(0, g.page_table[s], int(first[s]), block)[i] for s in range(n_seq)]).clone() for i in (0, 1)]

    for fn in ("step", "refresh"):
        g.tokens.copy_(tok0)
        g.mask.copy_(mask0)
        where = at.clone()
        if fn == "step":
            g.ctx.step_scored(g.tokens, g.mask, p, g.page_table, 0.9, 0, g.conf, g.argmax, g.n_committed, position=where)
        else:
            g.ctx.refresh_block_scored(g.tokens, p.clone(), g.page_table, position=where)
        torch.cuda.synchronize()
        assert torch.equal(where, at + (block if fn == "refresh" else 0))
        got = rows(p)
        g.tokens.copy_(tok0)
        g.mask.copy_(mask0)
        g.ctx.step(g.tokens, g.mask, at, g.page_table, 0.9, 0, g.conf, g.argmax, g.n_committed)
        torch.cuda.synchronize()
        want = rows(at)
        assert got[0].any() and all(torch.equal(a, b) for a, b in zip(got, want)), fn
    g.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n_seq,block,lo,hi,columns", [(1, 32, 100, 100, 40), (3, 13, 20, 900, 60), (2, 64, 1100, 1300, 96), (5, 64, 20, 200, 40)])
def test_scores_of_a_refresh(dtype, n_seq, block, lo, hi, columns):
    """A refresh leaves the scores of its block's queries: layer 0's from the definition, every layer's sum to one per query, and all are those that
    a step on the same tokens leaves."""
    cfg, w, inp, g = run_of(dtype, n_seq, block, lo, hi, 180 + n_seq, columns)
    torch = g.torch
    width = int(inp.prefix_len.max()) + block + 4
    old = torch.rand((cfg.n_layers, n_seq, cfg.n_heads, width), device=g.dev)
    scores, p = [torch.full_like(old, -1.0) for _ in range(2)], g.prefix_len.clone()
    tok0 = g.tokens.clone()
    g.ctx.refresh_block_scored(g.tokens, p, g.page_table, score_in=old, score_out=scores[0], decay=0.5)
    assert torch.equal(p, g.prefix_len + block) and torch.equal(g.tokens, tok0)
    g.ctx.step_scored(g.tokens, g.mask, g.prefix_len, g.page_table, 0.9, 0, g.conf, g.argmax, g.n_committed, score_in=old, score_out=scores[1],
                      decay=0.5)
    torch.cuda.synchronize()
    assert torch.equal(scores[0], scores[1])
    f64 = lambda a: (di.configs.bf16_to_f32(a) if a.dtype == np.uint16 else a).astype(np.float64)
    emb, wq, hd, nh = f64(w["emb"]), f64(w["layers"][0]["wq"]), cfg.head_dim, cfg.n_heads
    for s in range(n_seq):
        q0, n = int(inp.prefix_len[s]), int(inp.prefix_len[s]) + block
        gathered = (scores[0][:, s, :, :n].double() - 0.5 * old[:, s, :, :n].double()).cpu().numpy()
        assert (scores[0][:, s, :, n:] == -1).all()
        # weights: a few steps of 2^-24 each and of the old score; n of them
        assert np.abs(gathered.sum(-1) - block).max() <= block * 2.0 ** -14 + n * 2.0 ** -24
        x = emb[inp.block_tokens[s]]
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + cfg.rms_eps) * w["layers"][0]["attn_gain"]
        q = (x @ wq.T).reshape(block, nh, hd)
        ang = (q0 + np.arange(block))[:, None] * cfg.rope_theta ** (-2.0 * np.arange(hd // 2) / hd)
        cs, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
        q = np.concatenate([q[..., :hd // 2] * cs - q[..., hd // 2:] * sn, q[..., hd // 2:] * cs + q[..., :hd // 2] * sn], -1)
        k = g.read_kv(s, 0, 0, n)[0].astype(np.float64).reshape(-1, nh, hd)
        for h in range(nh):
            z = q[:, h] @ k[:, h].T / np.sqrt(hd)
            e = np.exp(z - z.max(-1, keepdims=True))
            ref = (e / e.sum(-1, keepdims=True)).sum(0)
            # queries are kept to 2^-16 (two bfloat16 planes) or float32: a score moves by at most that of sum |q k| scale
            bar = 2 * np.abs(q[:, h]).max() * np.abs(k[:, h]).max() * np.sqrt(hd) * 2.0 ** -14 + 2.0 ** -14
            assert np.abs(gathered[0, h] - ref).max() <= bar * ref.max() + 2.0 ** -24, (s, h)
    g.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n_seq,block,lo,hi,columns", [(2, 1, 1, 3, 4), (2, 32, 100, 900, 70), (3, 64, 20, 60, 12)])
def test_scored_step_and_refresh_captured(dtype, n_seq, block, lo, hi, columns):
    """A step with scores and a refresh with scores in one graph: every replay leaves what the eager calls left, with eager work on other tokens between
    the replays.  The score rows end in the block of the longest sequence."""
    cfg, w, inp, g = run_of(dtype, n_seq, block, lo, hi, 190 + n_seq, columns)
    torch = g.torch
    width = int(inp.prefix_len.max()) + block // 2
    state = dict(tokens=g.tokens, mask=g.mask, conf=g.conf, argmax=g.argmax, n=g.n_committed, length=g.prefix_len.clone(),
                 at=(g.prefix_len + 2).contiguous(), step=torch.zeros((cfg.n_layers, n_seq, cfg.n_heads, width), device=g.dev),
                 refresh=torch.zeros((cfg.n_layers, n_seq, cfg.n_heads, width), device=g.dev))
    start = {k: v.clone() for k, v in state.items()}
    kv0 = g.ctx.kv.clone()

    def run():
        g.ctx.step_scored(g.tokens, g.mask, state["length"], g.page_table, 0.02, 0, g.conf, g.argmax, g.n_committed, position=state["at"],
                          score_out=state["step"])
        g.ctx.refresh_block_scored(g.tokens, state["length"], g.page_table, position=state["at"], score_in=state["step"], score_out=state["refresh"],
                                   decay=0.9)

    def reset():
        for k, v in start.items():
            state[k].copy_(v)
        g.ctx.kv.copy_(kv0)

    run()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in state.items()}
    kv = g.ctx.kv.clone()
    assert want["refresh"].any() and torch.equal(want["at"], start["at"] + block)
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rep in range(4):
        reset()
        g.tokens.copy_((start["tokens"] + 7 * rep + 1) % (cfg.vocab - 1))
        run()
        torch.cuda.synchronize()
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in want.items():
            assert torch.equal(state[k], v), (rep, k)
        assert torch.equal(g.ctx.kv, kv), rep
    g.close()
