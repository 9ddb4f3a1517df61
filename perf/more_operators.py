"""Measured cases of the operators that search over several continuations on the paged cache: attention of new tokens under a
rule (`attend`: causal by blocks, prefix, window, documents, capped scores, distance bias), the choice of the best (row, token)
pairs of a sequence's hypotheses (`select`), sequences that fork from parents and share their pages (`fork`), and the move of
the pages in use to the front of the pool (`compact`).

The cache is the library's page pool, [layer][page][K | V][...]: the K part of a page holds, per head, blocks of 32
bytes of features with the page's 16 slots next to each other, the V part the page's 16 slots per head and feature.  The plain
forms index a tensor of that layout.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, **more):
    c = dict(name=name, op=op, dtype="bf16")
    if op == "attend":
        # heads of the cache, each with `group` query heads; len_min .. len_max new tokens behind past_min .. past_max cached ones,
        # both spread evenly; block 0: no order in time, 1: causal, more: causal by blocks; prefix: positions that all see;
        # document: length of the documents that do not see each other (0: one); cap: of the scores; slopes: bias by distance
        c.update(heads=16, group=1, head_dim=128, n_seq=1, len_min=1, len_max=1, past_min=511, past_max=511, block=1, prefix=0,
                 window=0, document=0, cap=0.0, slopes=False, lse=False)
    elif op == "select":
        # rows: hypotheses of a sequence, or their undecided positions; live: tenths of them that take part; held: some are finished
        c.update(n_seq=1, rows=8, vocab=157184, keep=8, live=10, held=False, banned=False)
    elif op == "fork":
        # prompts with old_beams sequences each, of which `survivors` have children; room: positions to reserve, rewrite: positions at
        # the end that will be written again
        c.update(heads=16, head_dim=128, layers=1, prompts=1, old_beams=1, survivors=1, new_beams=4, past_min=700, past_max=700,
                 room=32, rewrite=0)
    else:
        # sequences that hold a part of the pool: share tenths of its pages, scattered
        c.update(heads=16, head_dim=128, layers=1, n_seq=4, past_min=100, past_max=700, share=6)
    c.update(more)
    return c


def listed():
    return [
        # one token behind a short context, scores capped: the smallest call
        _case("attend_s1_p511_cap", "attend", cap=30.0),
        # a chunk of a long prompt, bidirectional prompt in front, blocks of the headline step's length
        _case("attend_chunk512_p4096_blocks", "attend", len_min=512, len_max=512, past_min=4096, past_max=4096, block=32, prefix=1000, lse=True),
        # a whole long prompt at once, causal, grouped query heads
        _case("attend_prompt8191_causal_g4", "attend", heads=8, group=4, len_min=8191, len_max=8191, past_min=0, past_max=0),
        # packed prompts: documents that do not see each other, capped
        _case("attend_prompts_documents_cap", "attend", n_seq=4, len_min=333, len_max=1811, past_min=0, past_max=0, block=0, document=301, cap=50.0),
        # many users, one token each, grouped query heads, bias by distance within a window
        _case("attend_b48_s1_slopes_window", "attend", heads=8, group=4, n_seq=48, past_min=1000, past_max=8000, window=4097, slopes=True,
              lse=True),
        # the float32 test model's heads: drafts behind odd contexts in a window with a prefix that stays
        _case("attend_f32_b3_window", "attend", dtype="f32", heads=4, head_dim=64, n_seq=3, len_min=5, len_max=333, past_min=64, past_max=901,
              window=200, prefix=17, slopes=True),
        # four beams of one sequence
        _case("select_b1_r4", "select", dtype="f32", rows=4, keep=4, held=True),
        # hypotheses of a batch, every undecided position a row
        _case("select_b8_r64_positions", "select", n_seq=8, rows=64, keep=16, live=6, banned=True),
        # the first fork behind one prompt
        _case("fork_b1_4", "fork"),
        # eight beams of eight prompts, half of them survive; the last 16 positions will be refreshed
        _case("fork_b8_8", "fork", layers=4, prompts=8, old_beams=8, survivors=4, new_beams=8, past_min=200, past_max=4001, room=32,
              rewrite=16),
        # the float32 test model's cache
        _case("compact_f32_b4", "compact", dtype="f32", heads=4, head_dim=64, layers=2),
        # a long-running pool
        _case("compact_b48", "compact", layers=2, n_seq=48, past_min=100, past_max=2000, share=6),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """A case of the listed ones' ranges that costs no more than the largest of its operator (a float32 product counts eight times)."""
    most = {}
    for c in listed():
        w = work(c)
        a = most.get(c["op"], w)
        most[c["op"]] = {k: max(a[k], w[k]) for k in w}
    while True:
        c = _draw(rng)
        if c["op"] == "attend":
            # (what the plain form's padded scores take)
            size = c["n_seq"] * c["heads"] * c["group"] * c["len_max"] * (c["len_max"] + c["past_max"])
            keys = c["n_seq"] * c["heads"] * c["head_dim"] * (c["len_max"] + c["past_max"])
            if size > 1 << 31 or keys > 1 << 29:
                continue
        w, a = work(c), most[c["op"]]
        if w["bytes"] <= a["bytes"] and w["flops"] * (8 if c["dtype"] == "f32" else 1) <= a["flops"]:
            return c


def _draw(rng):
    op = rng.choice(["attend", "attend", "attend", "select", "fork", "compact"])
    c = _case("", op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    del c["name"]
    if op == "attend":
        c["heads"], c["group"], c["head_dim"] = rng.choice([(16, 1, 128), (8, 4, 128), (4, 1, 64), (4, 2, 64), (5, 1, 64), (2, 8, 128), (3, 3, 64)])
        c["n_seq"] = _log_int(rng, 1, 48)
        c["len_max"] = _log_int(rng, 1, max(1, min(8191, 16384 // c["n_seq"])))
        c["len_min"] = rng.randint(1, c["len_max"])
        c["past_max"] = rng.choice([0, _log_int(rng, 1, 8000)])
        c["past_min"] = rng.randint(0, c["past_max"])
        c["block"] = rng.choice([0, 1, 1, 4, 32, 7])
        c["prefix"] = rng.choice([0, 0, _log_int(rng, 1, 2000)])
        c["window"] = rng.choice([0, 0, _log_int(rng, 1, 4097)])
        c["document"] = rng.choice([0, 0, _log_int(rng, 17, 3001)])
        c["cap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
        c["slopes"], c["lse"] = rng.random() < 0.4, rng.random() < 0.5
    elif op == "select":
        c["n_seq"] = _log_int(rng, 1, 16)
        c["rows"] = _log_int(rng, 1, 512 // c["n_seq"])
        c["vocab"] = rng.choice([157184, _log_int(rng, 100, 157184), 4096])
        c["keep"] = rng.randint(1, 32)
        c["live"], c["held"], c["banned"] = rng.randint(4, 10), rng.random() < 0.5, rng.random() < 0.5
    elif op == "fork":
        c["heads"], c["head_dim"] = rng.choice([(16, 128), (8, 128), (4, 64), (5, 64), (3, 64)])
        c["layers"] = rng.choice([1, 1, 2, 3, 4])
        c["prompts"] = _log_int(rng, 1, 8)
        c["old_beams"], c["new_beams"] = rng.randint(1, 8), rng.randint(1, 8)
        c["survivors"] = rng.randint(1, c["old_beams"])
        c["past_max"] = _log_int(rng, 1, 4001)
        c["past_min"] = rng.randint(0, c["past_max"])
        c["room"], c["rewrite"] = rng.randint(0, 80), rng.choice([0, 0, 16, 37])
    else:
        c["heads"], c["head_dim"] = rng.choice([(16, 128), (8, 128), (4, 64), (5, 64), (3, 64)])
        c["layers"] = rng.choice([1, 1, 2, 3, 4])
        c["n_seq"] = _log_int(rng, 1, 48)
        c["past_max"] = _log_int(rng, 1, 2000)
        c["past_min"] = rng.randint(0, c["past_max"])
        c["share"] = rng.randint(2, 10)
    return c


def _spread(n, lo, hi, turn):
    at = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]
    return [at[(i * turn + 3) % n] for i in range(n)] if math.gcd(turn, n) == 1 else at


def _pasts(c):
    return _spread(c["prompts"] if c["op"] == "fork" else c["n_seq"], c["past_min"], c["past_max"], 5)


def _ceil(a, b):
    return -(-a // b)


# ---------------------------------------------------------------------------------------------- inputs

class _Model:
    """What a context of the library is created from: the heads of the case in front of a small model."""
    hidden, n_experts, top_k, moe_inter, vocab, norm_topk = 64, 1, 1, 64, 64, 1
    mask_id, rms_eps, rope_theta, logit_scale = 63, 1e-5, 10000.0, 1.0

    def __init__(self, c):
        self.n_layers, self.n_heads, self.head_dim, self.dtype = c.get("layers", 1), c["heads"], c["head_dim"], c["dtype"]


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + 29)
    st = {"attend": _prepare_attend, "select": _prepare_select, "fork": _prepare_fork, "compact": _prepare_compact}[case["op"]](case, g)
    st["case"] = case
    if own:
        from paper_2510_08666_amd import binding
        if case["op"] == "select":
            st["scratch"] = binding.beam_scratch(case["n_seq"], case["rows"], case["vocab"], case["keep"])
        else:
            pool = st["pool"]
            st["ctx"] = binding.Context(_Model(case), pool.shape[1], 64, 64, st["max_pos"])
            st["pool"] = st["ctx"].kv.view(pool.dtype).view(pool.shape)
            st["pool"].copy_(pool)
    return st


def _pool(c, g, n_pages):
    shape = (c.get("layers", 1), n_pages, 2, c["heads"] * PAGE * c["head_dim"])
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(TYPES[c["dtype"]])


def _rows_of_pages(order, need, columns):
    """Page table rows of need[s] entries each, taken from `order` one after the other."""
    table = torch.zeros((len(need), columns), dtype=torch.int32, device=DEV)
    ends = np.cumsum([0] + need).tolist()
    for s, n in enumerate(need):
        table[s, :n] = order[ends[s]:ends[s + 1]]
    return table


def _attend_lens(c):
    return _spread(c["n_seq"], c["len_min"], c["len_max"], 7), _pasts(c)


def _prepare_attend(c, g):
    lens, past = _attend_lens(c)
    need = [_ceil(l + p, PAGE) for l, p in zip(lens, past)]
    n_pages, T, nq, hd, ns = sum(need) + 3, sum(lens), c["heads"] * c["group"], c["head_dim"], c["n_seq"]
    st = dict(lens=lens, past=past, d_past=_ints(past), max_pos=(max(need) + 1) * PAGE)
    st["table"] = _rows_of_pages(torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32), need, max(need) + 1)
    st["pool"] = _pool(c, g, n_pages)
    st["q"] = (1.5 * torch.randn((T, nq * hd), generator=g, device=DEV)).to(TYPES[c["dtype"]])
    st["out"] = torch.zeros((T, nq * hd), dtype=TYPES[c["dtype"]], device=DEV)
    st["lse"] = torch.zeros((T, nq), dtype=torch.float32, device=DEV) if c["lse"] else None
    st["prefix"] = _ints([c["prefix"]] * ns) if c["prefix"] else None
    st["first"] = st["end"] = None
    if c["document"]:
        at = _ints(np.concatenate([np.arange(p, p + l) for l, p in zip(lens, past)]).tolist())
        st["first"] = at // c["document"] * c["document"]
        st["end"] = st["first"] + c["document"]
    # slopes as they are spread over heads: halving from 1/2 down to 2^-8, times the distance in tokens
    st["slope"] = 2.0 ** (-8.0 * torch.arange(1, nq + 1, dtype=torch.float32, device=DEV) / nq) if c["slopes"] else None
    return st


def _live(c):
    """Rows of a sequence that take part, and those of them that are finished."""
    live = [(7 * r + 3) % 10 < c["live"] for r in range(c["rows"])]
    return live, [l and c["held"] and r % 8 == 5 % c["rows"] for r, l in enumerate(live)]


def _prepare_select(c, g):
    ns, R, V = c["n_seq"], c["rows"], c["vocab"]
    live, held = _live(c)
    # a model's logits: a wide bulk, a few tokens far above it
    z = 2.5 * torch.randn((ns, R, V), generator=g, device=DEV)
    z += 8.0 * (torch.rand((ns, R, V), generator=g, device=DEV) < 6.0 / V)
    if c["banned"]:
        z[:, :, torch.randperm(V, generator=g, device=DEV)[:V // 50]] = -math.inf
    score = -12.0 * torch.rand((ns, R), generator=g, device=DEV)
    score = torch.where(torch.tensor(live, device=DEV), score, -math.inf)
    hold = torch.where(torch.tensor(held, device=DEV), 2, -1).to(torch.int32).expand(ns, R).contiguous() if c["held"] else None
    i32 = torch.int32
    return dict(logits=z.to(TYPES[c["dtype"]]), score=score, hold=hold, row=torch.zeros((ns, c["keep"]), dtype=i32, device=DEV),
                token=torch.zeros((ns, c["keep"]), dtype=i32, device=DEV), best=torch.zeros((ns, c["keep"]), dtype=torch.float32, device=DEV))


def _fork_sizes(c):
    """Of every prompt: length, first column that its beams own, columns held by an old one, columns needed by a new one."""
    n = _pasts(c)
    first_own = [max(0, x - c["rewrite"]) // PAGE for x in n]
    shared = [max(0, f - 2) if c["old_beams"] > 1 else 0 for f in first_own]      # two pages behind the prompt are each beam's own
    held = [max(1, _ceil(x + c["room"], PAGE)) for x in n]
    return n, first_own, shared, held


def _fork_pages(c):
    n, first_own, shared, held = _fork_sizes(c)
    used = sum(s + c["old_beams"] * (h - s) for s, h in zip(shared, held))
    fresh = sum(c["new_beams"] * (_ceil(x + c["room"], PAGE) - f) for x, f in zip(n, first_own))
    return used, used + fresh + used // 8 + 8


def _prepare_fork(c, g):
    n, first_own, shared, held = _fork_sizes(c)
    used, n_pages = _fork_pages(c)
    P, B, N = c["prompts"], c["old_beams"], c["new_beams"]
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    columns = max(held) + 1
    table = torch.full((P * B, columns), -1, dtype=torch.int32, device=DEV)
    at = 0
    for p in range(P):
        table[p * B:(p + 1) * B, :shared[p]] = order[at:at + shared[p]]
        at += shared[p]
        table[p * B:(p + 1) * B, shared[p]:held[p]] = order[at:at + B * (held[p] - shared[p])].view(B, -1)
        at += B * (held[p] - shared[p])
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs.index_add_(0, table[table >= 0].long(), torch.ones(int((table >= 0).sum()), dtype=torch.int32, device=DEV))
    # the survivors of every prompt are others each time, their children in an order of their own
    alive = torch.argsort(torch.rand((P, B), generator=g, device=DEV), 1)[:, :c["survivors"]]
    child = torch.argsort(torch.rand((P, N), generator=g, device=DEV), 1) % c["survivors"]
    parent = (torch.gather(alive, 1, child) + torch.arange(P, device=DEV)[:, None] * B).view(-1).to(torch.int32)
    old = lambda x: _ints(x).repeat_interleave(B)
    history = columns * PAGE
    i32 = torch.int32
    empty = lambda *s: torch.zeros(s, dtype=i32, device=DEV)
    return dict(parent=parent, d_len=old(n), d_held=old(held), table=table, refs=refs, pool=_pool(c, g, n_pages), max_pos=columns * PAGE,
                history=torch.randint(0, 157184, (P * B, history), generator=g, device=DEV, dtype=i32),
                credit=torch.rand((P * B, 64), generator=g, device=DEV), new_history=empty(P * N, history),
                new_credit=torch.zeros((P * N, 64), device=DEV), new_table=empty(P * N, columns), new_len=empty(P * N),
                new_held=empty(P * N), new_refs=empty(n_pages), short=empty(1))


def _compact_sizes(c):
    held = [_ceil(x, PAGE) for x in _pasts(c)]
    return held, max(sum(held) * 10 // c["share"], sum(held)) + 3


def _compact_moves(c):
    """Pages in use that lie behind the front: the pages in use are spread evenly."""
    held, n_pages = _compact_sizes(c)
    used = _compact_used(c)
    return int((used >= sum(held)).sum())


def _compact_used(c):
    held, n_pages = _compact_sizes(c)
    return np.arange(sum(held), dtype=np.int64) * n_pages // max(1, sum(held))


def _prepare_compact(c, g):
    held, n_pages = _compact_sizes(c)
    used = torch.tensor(_compact_used(c), device=DEV)
    order = used[torch.randperm(len(used), generator=g, device=DEV)].to(torch.int32)
    columns = max(held) + 1
    table = _rows_of_pages(order, held, columns)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[used] = 1
    i32 = torch.int32
    empty = lambda *s: torch.zeros(s, dtype=i32, device=DEV)
    return dict(d_held=_ints(held), table=table, refs=refs, pool=_pool(c, g, n_pages), max_pos=columns * PAGE, new_table=empty(*table.shape),
                new_refs=empty(n_pages), moved=empty(2, n_pages), count=empty(2))


# ---------------------------------------------------------------------------------------------- plain forms

def _plain_attend(st):
    """All sequences at once, padded to the longest."""
    c = st["case"]
    nh, G, hd, ns = c["heads"], c["group"], c["head_dim"], c["n_seq"]
    nq, kb = nh * G, 32 // st["pool"].element_size()
    lens, past = torch.tensor(st["lens"], device=DEV), st["d_past"].long()
    total = lens + past
    Lm, Km = max(st["lens"]), max(l + p for l, p in zip(st["lens"], st["past"]))
    pages = st["table"][:, :_ceil(Km, PAGE)].long()
    K = st["pool"][0, :, 0].view(-1, nh, hd // kb, PAGE, kb)[pages]             # [ns][page][head][block][slot][feature]
    V = st["pool"][0, :, 1].view(-1, nh, hd, PAGE)[pages]                       # [ns][page][head][feature][slot]
    K = K.permute(0, 2, 1, 4, 3, 5).reshape(ns, nh, -1, hd)[:, :, :Km].float()
    V = V.permute(0, 2, 1, 4, 3).reshape(ns, nh, -1, hd)[:, :, :Km].float()
    tok = torch.arange(Lm, device=DEV)
    row = (torch.cumsum(lens, 0) - lens)[:, None] + tok.expand(ns, Lm)
    real = tok < lens[:, None]
    row = torch.where(real, row, 0)
    q = st["q"][row].float().view(ns, Lm, nh, G, hd).permute(0, 2, 3, 1, 4).reshape(ns, nh, G * Lm, hd)
    z = torch.matmul(q, K.transpose(2, 3).contiguous()).view(ns, nh, G, Lm, Km)
    z *= hd ** -0.5
    p = (past[:, None] + tok)[:, :, None]                                       # [ns][token][1]
    j = torch.arange(Km, device=DEV)
    if c["cap"]:
        z = c["cap"] * torch.tanh(z / c["cap"])
    if c["slopes"]:
        z -= st["slope"].view(1, nh, G, 1, 1) * (p - j).abs().float()[:, None, None]
    pre = st["prefix"].long()[:, None, None] if c["prefix"] else torch.zeros((ns, 1, 1), dtype=torch.long, device=DEV)
    see = (j < total[:, None, None]).expand(ns, Lm, Km)
    near = see
    if c["block"]:
        near = near & (j < torch.where(p < pre, pre, pre + ((p - pre) // c["block"] + 1) * c["block"]))
    if c["window"]:
        near = near & ((p - j).abs() < c["window"])
    see = see & (near | (j < pre))
    if c["document"]:
        see = see & (j >= st["first"].long()[row][:, :, None]) & (j < st["end"].long()[row][:, :, None])
    see = see[:, None, None]
    z = z.masked_fill_(~see, -math.inf)
    m = z.amax(-1, keepdim=True)
    z = torch.exp(z.sub_(torch.where(m == -math.inf, 0.0, m)))
    l = z.sum(-1, keepdim=True)
    o = torch.matmul(z.div_(torch.where(l == 0, 1.0, l)).view(ns, nh, G * Lm, Km), V)
    st["out"].copy_(o.view(ns, nh, G, Lm, hd).permute(0, 3, 1, 2, 4).reshape(ns, Lm, nq * hd)[real])
    if not c["lse"]:
        return {"out": st["out"]}
    st["lse"].copy_((m + l.log())[..., 0].permute(0, 3, 1, 2).reshape(ns, Lm, nq)[real])
    return {"out": st["out"], "lse": st["lse"]}


def _plain_select(st):
    c = st["case"]
    ns, R, V = c["n_seq"], c["rows"], c["vocab"]
    z = st["logits"].double()                                                   # neighbours in the order are close
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    x = st["score"].double()[..., None] + (z - (m + torch.exp(z - m).sum(-1, keepdim=True).log()))
    if c["held"]:
        hold = st["hold"].long()[..., None]
        only = torch.where(torch.arange(V, device=DEV) == hold, st["score"].double()[..., None], -math.inf)
        x = torch.where(hold >= 0, only, x)
    x = torch.where(st["score"][..., None] == -math.inf, -math.inf, x).view(ns, R * V)
    best, at = torch.sort(x, dim=-1, descending=True, stable=True)
    k = min(c["keep"], R * V)
    best, at = best[:, :k], at[:, :k]
    none = best == -math.inf
    st["row"].fill_(-1)[:, :k] = torch.where(none, -1, at // V).int()
    st["token"].fill_(-1)[:, :k] = torch.where(none, -1, at % V).int()
    st["best"].fill_(-math.inf)[:, :k] = best.float()
    return {"row": st["row"], "token": st["token"], "score": st["best"]}


def _plain_fork(st):
    c = st["case"]
    parent, refs, table = st["parent"].long(), st["refs"], st["table"].long()
    n, held = st["d_len"].long()[parent], st["d_held"].long()[parent]
    need, have, first_own = (n + c["room"] + PAGE - 1) // PAGE, (n + PAGE - 1) // PAGE, (n - c["rewrite"]).clamp(min=0) // PAGE
    col = torch.arange(table.shape[1], device=DEV)
    page = torch.where(col < held[:, None], table[parent], -1)
    same = parent[:, None] == parent[None]
    first = ~(same & (torch.arange(len(parent), device=DEV)[:, None] > torch.arange(len(parent), device=DEV))).any(1)
    share = col < first_own[:, None]
    take = ~share & (col < need[:, None]) & first[:, None] & (page >= 0) & (refs[page.clamp(min=0)] == 1)
    fresh = ~share & (col < need[:, None]) & ~take
    rank = (torch.cumsum(fresh.view(-1).int(), 0) - 1).view(fresh.shape).clamp(min=0)
    free = torch.sort((refs > 0).int(), stable=True)[1]
    st["short"].copy_((fresh.sum() - (refs <= 0).sum()).clamp(min=0))
    new = torch.where(share | take, page, torch.where(fresh, free[rank.clamp(max=len(free) - 1)], -1))
    st["new_table"].copy_(new)
    st["new_len"].copy_(n)
    st["new_held"].copy_(need)
    st["new_refs"].copy_(refs)
    out = table[col < st["d_held"][:, None]]
    st["new_refs"].index_add_(0, out, torch.full(out.shape, -1, dtype=torch.int32, device=DEV))
    into = new[new >= 0]
    st["new_refs"].index_add_(0, into, torch.ones(into.shape, dtype=torch.int32, device=DEV))
    copied = fresh & (col < have[:, None]) & (page >= 0)
    st["pool"][:, new[copied]] = st["pool"][:, page[copied]]
    st["new_history"].copy_(st["history"][parent])
    st["new_credit"].copy_(st["credit"][parent])
    return _fork_out(st)


def _fork_out(st):
    return {"table": st["new_table"], "len": st["new_len"], "held": st["new_held"], "refs": st["new_refs"], "short": st["short"],
            "history": st["new_history"], "credit": st["new_credit"], "pool": st["pool"]}


def _plain_compact(st):
    refs = st["refs"]
    n = len(refs)
    used, page = refs > 0, torch.arange(n, device=DEV)
    front = used.sum()
    mover = used & (page >= front)
    free = torch.sort(used.int(), stable=True)[1]
    to = torch.where(mover, free[(torch.cumsum(mover.int(), 0) - 1).clamp(min=0)], torch.where(used, page, -1))
    st["moved"][0] = to.int()
    st["moved"][1].fill_(-1)
    src = page[mover]
    st["moved"][1, :len(src)] = src.int()
    st["count"][0], st["count"][1] = front, len(src)
    st["new_refs"].zero_()
    st["new_refs"][to[used]] = refs[used]
    inside = torch.arange(st["table"].shape[1], device=DEV) < st["d_held"][:, None]
    st["new_table"].copy_(torch.where(inside, to[st["table"].long().clamp(min=0)], -1))
    st["pool"][:, to[src]] = st["pool"][:, src]
    return _compact_out(st)


def _compact_out(st):
    return {"table": st["new_table"], "refs": st["new_refs"], "moved": st["moved"], "count": st["count"], "pool": st["pool"]}


# ---------------------------------------------------------------------------------------------- the library's calls

def _own_attend(st):
    c = st["case"]
    st["ctx"].attend_ruled(0, st["lens"], st["d_past"], st["table"], st["q"], st["out"], block=c["block"], window=c["window"],
                           prefix=st["prefix"], first=st["first"], end=st["end"], cap=c["cap"], slope=st["slope"], lse=st["lse"])
    return {"out": st["out"], "lse": st["lse"]} if c["lse"] else {"out": st["out"]}


def _own_select(st):
    from paper_2510_08666_amd import binding
    binding.beam_select(st["logits"], st["score"], st["row"], st["token"], st["best"], st["scratch"], hold=st["hold"])
    return {"row": st["row"], "token": st["token"], "score": st["best"]}


def _own_fork(st):
    c = st["case"]
    st["ctx"].kv_fork(st["parent"], st["d_len"], st["d_held"], st["table"], st["refs"], st["new_len"], st["new_held"], st["new_table"],
                      st["new_refs"], st["short"], room=c["room"], rewrite=c["rewrite"],
                      states=[(st["history"], st["new_history"]), (st["credit"], st["new_credit"])])
    return _fork_out(st)


def _own_compact(st):
    st["ctx"].kv_compact(st["d_held"], st["table"], st["refs"], st["new_table"], st["new_refs"], st["moved"], st["count"])
    return _compact_out(st)


def run(state):
    op = state["case"]["op"]
    if own:
        return {"attend": _own_attend, "select": _own_select, "fork": _own_fork, "compact": _own_compact}[op](state)
    return {"attend": _plain_attend, "select": _plain_select, "fork": _plain_fork, "compact": _plain_compact}[op](state)


# ---------------------------------------------------------------------------------------------- work and exact values

def _visible(c, n, p0):
    """Per new token of a sequence: key ranges [a0, a1) and [b0, b1) that it sees (they do not overlap)."""
    p, total = np.arange(p0, p0 + n), p0 + n
    lo, hi = np.zeros(n, dtype=np.int64), np.full(n, total)
    if c["document"]:
        lo, hi = p // c["document"] * c["document"], np.minimum(hi, p // c["document"] * c["document"] + c["document"])
    pre = c["prefix"]
    b0, b1 = lo, hi
    if c["block"]:
        b1 = np.minimum(b1, np.where(p < pre, pre, pre + ((p - pre) // c["block"] + 1) * c["block"]))
    if c["window"]:
        b0, b1 = np.maximum(b0, p - c["window"] + 1), np.minimum(b1, p + c["window"])
    a1 = np.maximum(lo, np.minimum(pre, hi))
    b0 = np.maximum(b0, a1)
    return lo, a1, b0, np.maximum(b0, b1)


def _page_bytes(c):
    return 2 * PAGE * c["heads"] * c["head_dim"] * (2 if c["dtype"] == "bf16" else 4)


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "attend":
        nh, G, hd = c["heads"], c["group"], c["head_dim"]
        pairs = keys = 0
        for n, p0 in zip(*_attend_lens(c)):
            a0, a1, b0, b1 = _visible(c, n, p0)
            pairs += int((a1 - a0 + b1 - b0).sum())
            mark = np.zeros(n + p0 + 1, dtype=np.int64)
            for at, to in ((a0, a1), (b0, b1)):
                np.add.at(mark, at, 1)
                np.add.at(mark, to, -1)
            keys += int((np.cumsum(mark) > 0).sum())
        T = sum(_attend_lens(c)[0])
        return {"bytes": keys * 2 * nh * hd * es + 2 * T * nh * G * hd * es + (T * nh * G * 4 if c["lse"] else 0) + (8 * T if c["document"] else 0),
                "flops": 4 * pairs * nh * G * hd}
    if c["op"] == "select":
        live, held = _live(c)
        rows = c["n_seq"] * (sum(live) - sum(held))
        return {"bytes": rows * c["vocab"] * es + c["n_seq"] * (c["rows"] * 8 + c["keep"] * 12), "flops": 3 * rows * c["vocab"]}
    if c["op"] == "fork":
        n, first_own, shared, held = _fork_sizes(c)
        P, N = c["prompts"], c["new_beams"]
        copies = sum((N - min(N, c["survivors"])) * (_ceil(x, PAGE) - f) for x, f in zip(n, first_own))
        columns = max(held) + 1
        meta = 2 * P * N * (columns * 4 + columns * PAGE * 4 + 256) + 8 * _fork_pages(c)[1]
        return {"bytes": 2 * copies * c["layers"] * _page_bytes(c) + meta, "flops": 0}
    held, n_pages = _compact_sizes(c)
    return {"bytes": 2 * _compact_moves(c) * c["layers"] * _page_bytes(c) + n_pages * 16 + 8 * c["n_seq"] * (max(held) + 1), "flops": 0}


def exact(case, seed):
    c = case
    if c["op"] in ("fork", "compact"):
        return None               # copies and whole numbers
    if c["op"] == "attend" and work(c)["flops"] > 1 << 42:
        return None
    st = prepare(case, seed)
    f64 = torch.float64
    if c["op"] == "select":
        best = torch.full((c["n_seq"], c["keep"]), -math.inf, dtype=f64, device=DEV)
        for s in range(c["n_seq"]):
            found = []
            for r in range(c["rows"]):
                base = float(st["score"][s, r])
                if base == -math.inf:
                    continue
                if c["held"] and int(st["hold"][s, r]) >= 0:
                    found.append(torch.tensor([base], dtype=f64, device=DEV))
                    continue
                x = torch.log_softmax(st["logits"][s, r].to(f64), 0) + base
                found.append(torch.topk(x, min(c["keep"], c["vocab"]))[0])
            if found:
                x = torch.sort(torch.cat(found), descending=True)[0][:c["keep"]]
                best[s, :len(x)] = x
        return {"row": None, "token": None, "score": best}
    nh, G, hd, ns = c["heads"], c["group"], c["head_dim"], c["n_seq"]
    kb = 32 // st["pool"].element_size()
    outs, norms, t = [], [], 0
    for s in range(ns):
        n, p = st["lens"][s], st["past"][s]
        pages = st["table"][s, :_ceil(n + p, PAGE)].long()
        k = st["pool"][0, pages, 0].view(-1, nh, hd // kb, PAGE, kb).to(f64).transpose(2, 3).reshape(-1, nh, PAGE, hd)
        v = st["pool"][0, pages, 1].view(-1, nh, hd, PAGE).to(f64).transpose(2, 3)
        q = st["q"][t:t + n].to(f64).view(n, nh * G, hd)
        key, at = torch.arange(n + p, device=DEV), torch.arange(p, p + n, device=DEV)
        a0, a1, b0, b1 = (torch.tensor(x, device=DEV)[:, None] for x in _visible(c, n, p))
        hidden = ~(((key >= a0) & (key < a1)) | ((key >= b0) & (key < b1)))
        away = (key[None] - at[:, None]).abs().to(f64)
        o, e = torch.zeros((n, nh * G, hd), dtype=f64, device=DEV), torch.zeros((n, nh * G), dtype=f64, device=DEV)
        for h in range(nh * G):
            kh, vh = (y[:, h // G].reshape(-1, hd)[:n + p] for y in (k, v))
            z = q[:, h] @ kh.t() / math.sqrt(hd)
            if c["cap"]:
                z = (z / c["cap"]).tanh() * c["cap"]
            if c["slopes"]:
                z = z - st["slope"][h].to(f64) * away
            z = z.masked_fill(hidden, -math.inf)
            e[:, h] = torch.logsumexp(z, -1)
            o[:, h] = torch.nan_to_num(torch.softmax(z, -1)) @ vh
        outs.append(o.reshape(n, nh * G * hd))
        norms.append(e)
        t += n
    return {"out": torch.cat(outs), "lse": torch.cat(norms)} if c["lse"] else {"out": torch.cat(outs)}
