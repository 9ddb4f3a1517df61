"""A search over several continuations of a prompt, as a program runs it: the hypotheses share the prompt's pages, the best (position, token)
pairs go on, the pool is packed, and what they compute is what hypotheses with caches of their own compute."""
import math

import pytest
import torch

import dinfer_inputs as di

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32


@pytest.mark.parametrize("dtype,P,S,B", [("f32", 37, 16, 3), ("bf16", 64, 13, 4)])
def test_hypotheses_of_a_block(dtype, P, S, B):
    import search_ops as ops
    from harness import make_case
    from paper_2510_08666_amd import binding as b
    cfg = di.configs.scaled(di.model_preset("tiny"), dtype=dtype, n_layers=2)
    cfg, w, _ = make_case(di.Workload("search", cfg, 1, S, P, P, seed_index=31))
    g = torch.Generator().manual_seed(P)
    prompt = torch.randint(0, cfg.vocab - 1, (P,), generator=g).to(I32).to(DEV)
    columns, n_pages = 9, 64
    ctx = b.Context(cfg, n_pages, 8, 128, columns * 16)
    ctx.load_weights(w)
    alone = b.Context(cfg, 60, 8, 128, columns * 16, weights_buffer=ctx.weights)
    for c in (ctx, alone):
        c.kv.zero_()
    i32 = lambda *s: torch.zeros(s, dtype=I32, device=DEV)

    def fork(parent, length, held, table, refs, **kw):
        n = len(parent)
        out = [i32(n), i32(n), i32(n, columns), i32(n_pages), i32(1)]
        ctx.kv_fork(torch.tensor(parent, dtype=I32, device=DEV), length, held, table, refs, *out, **kw)
        assert out[4].item() == 0
        return out[:4]

    # pages for the prompt, the prompt, its hypotheses
    length, held, table, refs = fork([-1], None, None, None, i32(n_pages) + (torch.arange(n_pages, device=DEV) % 3 == 1).to(I32), room=P)
    others = refs - (torch.bincount(table[0, :held[0]].long(), minlength=n_pages)).to(I32)      # (pages of somebody else's)
    length.fill_(P)
    ctx.prefill(prompt, [P], table)
    length, held, table, refs = fork([0] * B, length, held, table, refs, room=S)
    shared = P // 16
    assert all((table[:, c] == table[0, c]).all() and refs[table[0, c].long()] == B for c in range(shared))
    own = table[:, shared:int(held[0])]
    assert len(set(own.flatten().tolist())) == own.numel()
    tokens, score = torch.full((B, S), cfg.mask_id, dtype=I32, device=DEV), torch.tensor([0.0] + [-math.inf] * (B - 1))
    conf, argmax, done = torch.zeros(B, S, device=DEV), i32(B, S), i32(B)
    none = torch.zeros(B, dtype=torch.int64, device=DEV)
    scratch = b.beam_scratch(1, B * S, cfg.vocab, B)
    row, token, best = i32(1, B), i32(1, B), torch.zeros(1, B, device=DEV)
    for turn in range(4):
        ctx.step(tokens.clone(), none.clone(), length, table, 0.5, 0, conf, argmax, done)      # (an empty mask: a forward that commits nothing)
        logits = ctx.debug_logits(B * S).view(1, B * S, -1)
        base = torch.where(tokens.cpu() == cfg.mask_id, score[:, None], -math.inf).reshape(1, B * S)
        b.beam_select(logits, base.to(DEV), row, token, best, scratch)
        torch.cuda.synchronize()
        want = ops.select(logits.cpu(), base, B)[0]
        assert [x[1:] for x in want] == list(zip(row[0].tolist(), token[0].tolist()))
        parent, at = [r // S for r in row[0].tolist()], [r % S for r in row[0].tolist()]
        new = torch.zeros_like(tokens)
        length, held, table, refs = fork(parent, length, held, table, refs, room=S, states=[(tokens, new)])
        assert torch.equal(new, tokens[torch.tensor(parent, device=DEV)])
        tokens, score = new, best[0].cpu()
        tokens[torch.arange(B), torch.tensor(at)] = token[0]
        assert torch.equal(refs - others, torch.bincount(torch.cat([table[i, :held[i]] for i in range(B)]).long(), minlength=n_pages).to(I32))
    # the block as it stands is decided, the pool packed, the next block begins
    tokens = torch.where(tokens == cfg.mask_id, 7, tokens).to(I32)
    ctx.refresh_block(tokens, length, table)
    length, held, table, refs = fork(list(range(B)), length, held, table, refs, room=S)
    packed, count = [i32(B, columns), i32(n_pages), i32(2, n_pages)], i32(2)
    ctx.kv_compact(held, table, refs, *packed, count)
    table, refs = packed[:2]
    assert (refs[:count[0]] > 0).all() and (refs[count[0]:] == 0).all()
    # hypotheses with caches of their own
    table2 = torch.randperm(60, generator=g)[:B * columns].view(B, columns).to(I32).to(DEV)
    for i in range(B):
        alone.prefill(prompt, [P], table2[i:i + 1])
    length2 = torch.full((B,), P, dtype=I32, device=DEV)
    alone.refresh_block(tokens, length2, table2)
    assert torch.equal(length, length2)
    outs = []
    for c, t in ((ctx, table), (alone, table2)):
        block, mask = torch.full((B, S), cfg.mask_id, dtype=I32, device=DEV), torch.full((B,), (1 << S) - 1, dtype=torch.int64, device=DEV)
        conf, argmax, done = torch.zeros(B, S, device=DEV), i32(B, S), i32(B)
        c.step(block, mask, length, t, 0.3, 0, conf, argmax, done)
        q = torch.randn(B * S, cfg.n_heads * cfg.head_dim, generator=torch.Generator().manual_seed(1)).to(DEV).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        out = torch.zeros_like(q)
        c.attend_ruled(1, [S] * B, length, t, q, out, block=S, prefix=length, window=50, cap=20.0)
        torch.cuda.synchronize()
        outs.append((conf, argmax, done, block, mask, out))
    for x, y in zip(*outs):
        assert torch.equal(x, y)
    ctx.close()
    alone.close()
