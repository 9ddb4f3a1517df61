"""Measured cases of the paged cache's operators: the pass that norms, rotates and stores a layer's queries, keys and
values (`append`), attention of new tokens over the cache under visibility words (`attend`), the attention weight that
cached positions gather (`score`), and the move of the positions worth keeping into other pages (`evict`).

The cache is the library's page pool, [layer][page][K | V][...]: the K part of a page holds, per head, blocks of 32
bytes of features with the page's 16 slots next to each other, the V part the page's 16 slots per head and feature.  The plain
forms index a tensor of that layout.
"""
import math

import torch

own = False

PAGE = 16
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, **more):
    """heads: heads of the cache, each with `group` query heads.  len_min .. len_max: new tokens of the sequences,
    past_min .. past_max: positions cached in front of them, both spread evenly over their range."""
    c = dict(name=name, op=op, dtype="bf16", heads=16, group=1, head_dim=128, n_seq=1, len_min=32, len_max=32,
             past_min=512, past_max=512)
    if op == "append":
        c.update(norm=True, rotary_dim=128, interleaved=False, scaling="plain", factor=1.0)
    if op in ("attend", "score"):
        c.update(tree=False, lse=False)
    if op == "score":
        c.update(decay=1.0)
    if op == "evict":
        c.update(layers=1, keep=256, sink=4, recent=32)
    c.update(more)
    return c


def listed():
    return [
        # one block of the headline step: 32 tokens of one sequence, whole heads rotated in halves, head norms
        _case("append_b1_s32", "append"),
        # drafts of a batch: ragged lengths on odd positions, half of each head rotated in neighbouring pairs, ramped frequencies
        _case("append_b16_ragged_pairs", "append", heads=8, group=4, n_seq=16, len_min=1, len_max=64, past_min=200, past_max=7001,
              rotary_dim=64, interleaved=True, scaling="yarn", factor=4.0),
        # prompts of a batch, whole pages at a time
        _case("append_prompts", "append", n_seq=4, len_min=333, len_max=1811, past_min=0, past_max=0, scaling="ntk", factor=2.0),
        # one token behind a short context: the smallest call
        _case("attend_b1_s1_p512", "attend", len_min=1, len_max=1, past_min=511, past_max=511),
        # a long context under a tree of 64 drafts
        _case("attend_b1_s64_p4096_tree", "attend", len_min=64, len_max=64, past_min=4096, past_max=4096, tree=True, lse=True),
        # batched serving: ragged contexts on scattered pages, odd draft counts
        _case("attend_b16_tree", "attend", n_seq=16, len_min=17, len_max=32, past_min=256, past_max=2048, tree=True),
        # many users with grouped query heads, several query tiles per cache head
        _case("attend_b48_g4", "attend", heads=8, group=4, n_seq=48, len_min=31, len_max=64, past_min=1000, past_max=8000, tree=True,
              lse=True),
        # the float32 test model's heads
        _case("attend_f32_b3", "attend", dtype="f32", heads=4, head_dim=64, n_seq=3, len_min=5, len_max=33, past_min=64, past_max=901),
        # weights of one block's queries, nothing known of their normalisers
        _case("score_b1_s32_p700", "score", past_min=700, past_max=700, decay=0.9),
        # a batch behind its attention, which left the normalisers
        _case("score_b16_lse", "score", n_seq=16, len_min=17, len_max=32, past_min=256, past_max=4096, tree=True, lse=True),
        # one sequence: a quarter of 701 positions stays
        _case("evict_b1_p701", "evict", past_min=701, past_max=701, keep=175),
        # a batch at the edge of its memory, two layers at a time
        _case("evict_b16_p4096", "evict", layers=2, n_seq=16, past_min=900, past_max=4096, keep=1024, sink=16, recent=64),
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
        w, a = work(c), most[c["op"]]
        if w["bytes"] <= a["bytes"] and w["flops"] * (8 if c["dtype"] == "f32" else 1) <= a["flops"]:
            return c


def _draw(rng):
    op = rng.choice(["append", "attend", "score", "evict"])
    heads, group, head_dim = rng.choice([(16, 1, 128), (8, 4, 128), (4, 1, 64), (4, 2, 64), (5, 1, 64), (2, 8, 128), (3, 3, 64)])
    c = _case("", op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), heads=heads, group=group, head_dim=head_dim)
    del c["name"]
    c["n_seq"] = _log_int(rng, 1, 48)
    if op == "append":
        longest = _log_int(rng, 1, max(1, min(1811, 4096 // c["n_seq"])))
        c.update(norm=rng.random() < 0.7, interleaved=rng.random() < 0.5, scaling=rng.choice(["plain", "linear", "ntk", "yarn"]),
                 factor=rng.choice([1.5, 2.0, 4.0, 8.0]), rotary_dim=rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4, 20]),
                 past_max=_log_int(rng, 1, 8000))
        if c["scaling"] == "plain":
            c["factor"] = 1.0
    else:
        longest = _log_int(rng, 1, 64)
        most = 8000 if c["dtype"] == "bf16" else 2000
        c["past_max"] = _log_int(rng, 1, min(most, 400000 // (c["n_seq"] * (1 if c["dtype"] == "bf16" else 4))))
    c["len_max"] = longest
    c["len_min"] = rng.randint(1, longest)
    c["past_min"] = rng.randint(0, c["past_max"])
    if op in ("attend", "score"):
        c.update(tree=rng.random() < 0.6, lse=rng.random() < 0.5)
    if op == "score":
        c["decay"] = rng.choice([1.0, 0.9, 0.5])
    if op == "evict":
        c["past_max"] = max(c["past_max"], 8)
        c["past_min"] = max(1, c["past_min"])
        c["layers"] = rng.choice([1, 1, 2, 3])
        c["keep"] = _log_int(rng, 1, c["past_max"])
        c["sink"] = rng.randint(0, min(8, c["keep"]))
        c["recent"] = rng.randint(0, c["keep"] - c["sink"])
    return c


def _spread(n, lo, hi, turn):
    at = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]
    return [at[(i * turn + 3) % n] for i in range(n)] if math.gcd(turn, n) == 1 else at


def _lens(c):
    """New tokens and cached positions of every sequence."""
    return _spread(c["n_seq"], c["len_min"], c["len_max"], 7), _spread(c["n_seq"], c["past_min"], c["past_max"], 5)


def _layers(c):
    return c.get("layers", 1)


# ---------------------------------------------------------------------------------------------- inputs

class _Model:
    """What a context of the library is created from: the heads of the case in front of a small model."""
    hidden, n_experts, top_k, moe_inter, vocab, norm_topk = 64, 1, 1, 64, 64, 1
    mask_id, rms_eps, rope_theta, logit_scale = 63, 1e-5, 10000.0, 1.0

    def __init__(self, c):
        self.n_layers, self.n_heads, self.head_dim, self.dtype = _layers(c), c["heads"], c["head_dim"], c["dtype"]


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _frequencies(c):
    """Angle per position of every pair, and the factor on cosine and sine (float64)."""
    r, theta = c["rotary_dim"], 10000.0
    j = torch.arange(r // 2, dtype=torch.float64, device=DEV)
    if c["scaling"] == "ntk":
        theta = theta * c["factor"] ** (r / (r - 2))
    f = theta ** (-2.0 * j / r)
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "yarn":
        corner = lambda turns: r * math.log(ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(theta))
        low, high = max(0, math.floor(corner(32.0))), min(r - 1, math.ceil(corner(1.0)))
        ramp = ((j - low) / max(high - low, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / c["factor"] * ramp, 0.1 * math.log(c["factor"]) + 1.0
    return f, 1.0


ORIGINAL = 2048     # positions that the ramped frequencies stretch


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + 17)
    dt, nh, hd, nq = TYPES[c["dtype"]], c["heads"], c["head_dim"], c["heads"] * c["group"]
    lens, past = _lens(c)
    ns, L, T = c["n_seq"], _layers(c), sum(lens)
    if c["op"] == "evict":
        lens = [0] * ns
    total = [l + p for l, p in zip(lens, past)]
    need = [-(-t // PAGE) for t in total]
    stride = max(need) + 1
    keep_pages = -(-c["keep"] // PAGE) if c["op"] == "evict" else 0
    n_pages = sum(need) + 3 + ns * keep_pages
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros((ns, stride), dtype=torch.int32, device=DEV)
    at = 0
    for s in range(ns):
        table[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
    # keys as a norm per head leaves them, a few of them in every direction's favour; values of unit size
    pool = _randn(g, L, n_pages, 2, nh * PAGE * hd).to(dt)
    st = dict(case=c, lens=lens, past=past, table=table, d_past=torch.tensor(past, dtype=torch.int32, device=DEV), pool=pool)
    if c["op"] == "append":
        st["qkv"] = (2.0 * _randn(g, T, (nq + 2 * nh) * hd)).to(dt)
        st["q_gain"] = 1 + 0.1 * _randn(g, hd) if c["norm"] else None
        st["k_gain"] = 1 + 0.1 * _randn(g, hd) if c["norm"] else None
        # positions as drafts have them: a few tokens share one
        back = torch.randint(0, 3, (T,), generator=g, device=DEV, dtype=torch.int32)
        pos = torch.cat([torch.arange(p, p + l, device=DEV, dtype=torch.int32) for l, p in zip(lens, past)])
        st["positions"] = (pos - back).clamp(min=0)
        st["q_out"] = torch.zeros((T, nq * hd), dtype=dt, device=DEV)
        st["max_pos"] = max(total) + 16
    elif c["op"] in ("attend", "score"):
        st["q"] = (1.5 * _randn(g, T, nq * hd)).to(dt)
        st["out"] = torch.zeros((T, nq * hd), dtype=dt, device=DEV)
        st["lse"] = torch.zeros((T, nq), dtype=torch.float32, device=DEV)
        st["visible"] = None
        if c["tree"]:
            # every draft sees itself and its ancestors; now and then one starts a branch of its own
            r = torch.randint(0, 1 << 20, (T,), generator=g, device=DEV).cpu().tolist()
            words, at = [], 0
            for l in lens:
                seen = []
                for i in range(l):
                    parent = i - 1 - r[at + i] % 4
                    seen.append((1 << i) | (seen[parent] if parent >= 0 else 0))
                words += [w - (1 << 64) if w >> 63 else w for w in seen]
                at += l
            st["visible"] = torch.tensor(words, dtype=torch.int64, device=DEV)
        if c["op"] == "score":
            width = max(total) + 5
            st["score_in"] = _randn(g, ns, nh, width).abs()
            st["score_out"] = torch.zeros_like(st["score_in"])
            if c["lse"]:
                parts = [_scores(st, s) for s in range(ns)]
                st["lse"] = torch.cat([torch.logsumexp(p, -1).permute(2, 0, 1).reshape(p.shape[2], nq) for p in parts])
    else:
        width = max(past) + 7
        score = _randn(g, L, ns, nh, width).abs()
        # positions that nobody looked at tie at zero, some others at a coarse grid
        u = torch.rand(score.shape, generator=g, device=DEV)
        score = torch.where(u < 0.2, torch.zeros_like(score), torch.where(u < 0.5, (score * 8).round() / 8, score))
        st["score"] = score
        st["score_out"] = torch.zeros_like(score)
        st["new_table"] = order[sum(need):sum(need) + ns * keep_pages].reshape(ns, keep_pages).contiguous()
        st["kept"] = torch.zeros((L, ns, nh, c["keep"]), dtype=torch.int32, device=DEV)
        st["new_len"] = torch.zeros(ns, dtype=torch.int32, device=DEV)
    if own:
        from paper_2510_08666_amd import binding
        st["ctx"] = binding.Context(_Model(c), n_pages, ns, 64, st.get("max_pos", stride * PAGE))
        st["ctx"].kv.view(dt).copy_(pool.view(-1))
        st["pool"] = st["ctx"].kv.view(dt).view(pool.shape)
        if c["op"] == "append":
            st["rotary"] = binding.rotary(c["rotary_dim"], interleaved=c["interleaved"], theta=10000.0, scaling=c["scaling"],
                                          factor=c["factor"], original_positions=ORIGINAL)
            st["rotary_table"] = binding.rotary_table(st["rotary"], st["max_pos"])
    elif c["op"] == "append":
        f, size = _frequencies(c)
        angle = torch.arange(st["max_pos"], dtype=torch.float64, device=DEV)[:, None] * f
        st["cos"], st["sin"] = (angle.cos() * size).float(), (angle.sin() * size).float()
    return st


# ---------------------------------------------------------------------------------------------- plain forms

def _views(pool, c):
    """K [page][head][block][slot][feature of block] and V [page][head][feature][slot] of one layer's pool."""
    nh, hd = c["heads"], c["head_dim"]
    kb = 32 // pool.element_size()
    return pool[:, 0].view(-1, nh, hd // kb, PAGE, kb), pool[:, 1].view(-1, nh, hd, PAGE)


def _rows(st, s, n, pool=None, of=("k", "v")):
    """Cached rows 0 .. n-1 of sequence s as [head][row][feature] in 32 bits."""
    c = st["case"]
    nh, hd = c["heads"], c["head_dim"]
    k, v = _views(st["pool"][0] if pool is None else pool, c)
    pages = st["table"][s, :-(-n // PAGE)].long()
    out = []
    if "k" in of:
        out.append(k[pages].permute(1, 0, 3, 2, 4).reshape(nh, -1, hd)[:, :n].float())
    if "v" in of:
        out.append(v[pages].permute(1, 0, 3, 2).reshape(nh, -1, hd)[:, :n].float())
    return out


def _seen(st, s):
    """[tokens][tokens]: which of the sequence's new keys its new tokens see (None: all)."""
    if st["visible"] is None:
        return None
    t0, n = sum(st["lens"][:s]), st["lens"][s]
    w = st["visible"][t0:t0 + n]
    return (w[:, None] >> torch.arange(n, device=DEV)) & 1 == 1


def _scores(st, s, k=None):
    """Masked scores [head][query head of the group][token][key]."""
    c = st["case"]
    nh, hd, G = c["heads"], c["head_dim"], c["group"]
    t0, n, p = sum(st["lens"][:s]), st["lens"][s], st["past"][s]
    k = _rows(st, s, p + n, of=("k",))[0] if k is None else k
    q = st["q"][t0:t0 + n].view(n, nh, G, hd).permute(1, 2, 0, 3).reshape(nh, G * n, hd).float().contiguous()
    z = torch.matmul(q, k.transpose(1, 2).contiguous()) * (hd ** -0.5)
    z = z.view(nh, G, n, p + n)
    seen = _seen(st, s)
    if seen is not None:
        z[..., p:] = z[..., p:].masked_fill(~seen, float("-inf"))
    return z


def _plain_append(st):
    c = st["case"]
    nh, hd, nq, r = c["heads"], c["head_dim"], c["heads"] * c["group"], c["rotary_dim"]
    T = st["qkv"].shape[0]
    x = st["qkv"].view(T, nq + 2 * nh, hd).float()
    q, k, v = x[:, :nq], x[:, nq:nq + nh], x[:, nq + nh:]
    if c["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-6) * st["q_gain"]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + 1e-6) * st["k_gain"]
    cos, sin = st["cos"][st["positions"].long()][:, None], st["sin"][st["positions"].long()][:, None]

    def turn(y):
        y = y.clone()
        a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
        na, nb = a * cos - b * sin, b * cos + a * sin
        if c["interleaved"]:
            y[..., 0:r:2], y[..., 1:r:2] = na, nb
        else:
            y[..., :r // 2], y[..., r // 2:r] = na, nb
        return y

    q, k = turn(q), turn(k)
    st["q_out"].copy_(q.reshape(T, nq * hd))
    K, V = _views(st["pool"][0], c)
    at = torch.cat([torch.arange(p, p + l, device=DEV) for l, p in zip(st["lens"], st["past"])])
    seq = torch.repeat_interleave(torch.arange(c["n_seq"], device=DEV), torch.tensor(st["lens"], device=DEV))
    page, slot = st["table"][seq, at // PAGE].long(), at % PAGE
    K[page, :, :, slot] = k.to(K.dtype).view(T, nh, K.shape[2], K.shape[4])
    V[page, :, :, slot] = v.to(V.dtype)
    return {"q": st["q_out"], "pool": st["pool"]}


def _plain_attend(st):
    c = st["case"]
    nh, hd, G = c["heads"], c["head_dim"], c["group"]
    for s in range(c["n_seq"]):
        t0, n, p = sum(st["lens"][:s]), st["lens"][s], st["past"][s]
        k, v = _rows(st, s, p + n)
        z = _scores(st, s, k)
        m = z.amax(-1, keepdim=True)
        e = torch.exp(z - m)
        l = e.sum(-1, keepdim=True)
        o = torch.matmul((e / l).view(nh, G * n, p + n), v.contiguous())
        st["out"][t0:t0 + n] = o.view(nh, G, n, hd).permute(2, 0, 1, 3).reshape(n, nh * G * hd).to(st["out"].dtype)
        if c["lse"]:
            st["lse"][t0:t0 + n] = (m + l.log())[..., 0].permute(2, 0, 1).reshape(n, nh * G)
    return {"out": st["out"], "lse": st["lse"]} if c["lse"] else {"out": st["out"]}


def _plain_score(st):
    c = st["case"]
    nh, G = c["heads"], c["group"]
    for s in range(c["n_seq"]):
        t0, n = sum(st["lens"][:s]), st["lens"][s]
        z = _scores(st, s)
        if c["lse"]:
            w = torch.exp(z - st["lse"][t0:t0 + n].view(n, nh, G).permute(1, 2, 0)[..., None])
        else:
            e = torch.exp(z - z.amax(-1, keepdim=True))
            w = e / e.sum(-1, keepdim=True)
        total = z.shape[-1]
        st["score_out"][s, :, :total] = c["decay"] * st["score_in"][s, :, :total] + w.sum((1, 2))
    return {"score": st["score_out"]}


def _plain_evict(st):
    c = st["case"]
    nh, hd, keep, ns = c["heads"], c["head_dim"], c["keep"], c["n_seq"]
    st["kept"].fill_(-1)
    st["score_out"].zero_()
    slot = torch.arange(keep, device=DEV)
    for layer in range(c["layers"]):
        K, V = _views(st["pool"][layer], c)
        for s in range(ns):
            n = st["past"][s]
            m = min(n, keep)
            x = st["score"][layer, s, :, :n].clone()
            x[:, :min(n, c["sink"])] = float("inf")
            x[:, max(0, n - c["recent"]):] = float("inf")
            idx = torch.sort(x, dim=-1, descending=True, stable=True)[1][:, :m]
            idx = torch.sort(idx, dim=-1)[0]
            st["kept"][layer, s, :, :m] = idx.int()
            st["score_out"][layer, s, :, :m] = torch.gather(st["score"][layer, s], 1, idx)
            page, new = st["table"][s][idx // PAGE].long(), st["new_table"][s][slot[:m] // PAGE].long()
            h = torch.arange(nh, device=DEV)[:, None]
            K[new[None, :], h, :, (slot[:m] % PAGE)[None, :]] = K[page, h, :, idx % PAGE]
            V[new[None, :], h, :, (slot[:m] % PAGE)[None, :]] = V[page, h, :, idx % PAGE]
    st["new_len"].copy_(st["d_past"].clamp(max=keep))
    return {"kept": st["kept"], "score": st["score_out"], "len": st["new_len"], "pool": st["pool"]}


# ---------------------------------------------------------------------------------------------- the library's calls

def _own(st):
    c, ctx = st["case"], st["ctx"]
    if c["op"] == "append":
        nq, nh, hd = c["heads"] * c["group"], c["heads"], c["head_dim"]
        q, k, v = st["qkv"].split([nq * hd, nh * hd, nh * hd], 1)
        ctx.kv_append(0, st["lens"], st["d_past"], st["table"], q, k, v, st["q_out"], q_gain=st["q_gain"], k_gain=st["k_gain"],
                      eps=1e-6, rotary=st["rotary"], rotary_table=st["rotary_table"], positions=st["positions"])
        return {"q": st["q_out"], "pool": st["pool"]}
    if c["op"] == "attend":
        ctx.attend(0, st["lens"], st["d_past"], st["table"], st["q"], st["out"], visible=st["visible"],
                   lse=st["lse"] if c["lse"] else None)
        return {"out": st["out"], "lse": st["lse"]} if c["lse"] else {"out": st["out"]}
    if c["op"] == "score":
        ctx.kv_score(0, st["lens"], st["d_past"], st["table"], st["q"], st["score_out"], score_in=st["score_in"], decay=c["decay"],
                     visible=st["visible"], lse=st["lse"] if c["lse"] else None)
        return {"score": st["score_out"]}
    ctx.kv_evict(0, c["layers"], c["keep"], c["sink"], c["recent"], st["score"], st["d_past"], st["table"], st["new_table"],
                 st["kept"], st["new_len"], score_out=st["score_out"])
    return {"kept": st["kept"], "score": st["score_out"], "len": st["new_len"], "pool": st["pool"]}


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "attend": _plain_attend, "score": _plain_score, "evict": _plain_evict}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------- work and exact values

def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    nh, G, hd = c["heads"], c["group"], c["head_dim"]
    lens, past = _lens(c)
    T, D = sum(lens), nh * hd
    if c["op"] == "append":
        row = (G + 2) * D
        return {"bytes": 2 * T * row * es + T * (c["rotary_dim"] * 4 + 4), "flops": T * (G + 1) * D * (7 if c["norm"] else 3)}
    if c["op"] == "evict":
        kept = sum(min(p, c["keep"]) for p in past)
        # every score read, the kept rows (K and V), their scores and indices moved
        return {"bytes": c["layers"] * (nh * sum(past) * 4 + kept * (2 * 2 * D * es + 2 * nh * 4)), "flops": 0}
    keys = sum(l + p for l, p in zip(lens, past))
    pairs = sum(l * (l + p) for l, p in zip(lens, past)) * nh * G
    words = T * 8 if c["tree"] else 0
    if c["op"] == "attend":
        return {"bytes": keys * 2 * D * es + T * G * D * 2 * es + words + (T * nh * G * 4 if c["lse"] else 0), "flops": 4 * pairs * hd}
    return {"bytes": keys * D * es + T * G * D * es + words + keys * nh * 8 + (T * nh * G * 4 if c["lse"] else 0), "flops": 2 * pairs * hd}


def exact(case, seed):
    c = case
    if c["op"] == "evict":
        return None               # copies and whole numbers
    nh, G, hd, ns = c["heads"], c["group"], c["head_dim"], c["n_seq"]
    nq = nh * G
    lens, past = _lens(c)
    if c["op"] != "append" and sum(l * (l + p) for l, p in zip(lens, past)) * nq * hd > 1 << 36:
        return None
    st = prepare(case, seed)
    f64 = torch.float64
    kb = 32 // st["pool"].element_size()
    if c["op"] == "append":
        T, r = sum(lens), c["rotary_dim"]
        x = st["qkv"].to(f64).view(T, nq + 2 * nh, hd)
        if c["norm"]:
            gain = torch.ones((nq + 2 * nh, hd), dtype=f64, device=DEV)
            gain[:nq], gain[nq:nq + nh] = st["q_gain"].to(f64), st["k_gain"].to(f64)
            size = (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
            size[:, nq + nh:] = 1
            x = x / size * gain
        f, factor = _frequencies(c)
        turned = torch.polar(torch.full((T, r // 2), factor, dtype=f64, device=DEV), st["positions"].to(f64)[:, None] * f)
        pairs = torch.arange(r, device=DEV).view(-1, 2) if c["interleaved"] else torch.arange(r, device=DEV).view(2, -1).t()
        y = torch.complex(x[:, :nq + nh, pairs[:, 0]], x[:, :nq + nh, pairs[:, 1]]) * turned[:, None]
        x = x.clone()
        x[:, :nq + nh, pairs[:, 0]], x[:, :nq + nh, pairs[:, 1]] = y.real, y.imag
        pool = st["pool"].to(f64)
        K, V = pool[0, :, 0].view(-1, nh, hd // kb, PAGE, kb), pool[0, :, 1].view(-1, nh, hd, PAGE)
        t = 0
        for s in range(ns):
            row = st["table"][s].tolist()
            for p0 in range(past[s] // PAGE * PAGE, past[s] + lens[s], PAGE):
                a, b = max(p0, past[s]), min(p0 + PAGE, past[s] + lens[s])
                part = x[t + a - past[s]:t + b - past[s]]
                K[row[p0 // PAGE], :, :, a - p0:b - p0] = part[:, nq:nq + nh].reshape(b - a, nh, hd // kb, kb).permute(1, 2, 0, 3)
                V[row[p0 // PAGE], :, :, a - p0:b - p0] = part[:, nq + nh:].permute(1, 2, 0)
            t += lens[s]
        return {"q": x[:, :nq].reshape(T, nq * hd), "pool": pool}
    outs, norms, scores = [], [], (st["score_out"].to(f64) if c["op"] == "score" else None)
    t = 0
    for s in range(ns):
        n, p = lens[s], past[s]
        total = n + p
        pages = st["table"][s, :-(-total // PAGE)].long()
        k = st["pool"][0, pages, 0].view(-1, nh, hd // kb, PAGE, kb).to(f64).transpose(2, 3).reshape(-1, nh, PAGE, hd)
        v = st["pool"][0, pages, 1].view(-1, nh, hd, PAGE).to(f64).transpose(2, 3)
        q = st["q"][t:t + n].to(f64).view(n, nq, hd)
        hidden = torch.zeros((n, total), dtype=torch.bool, device=DEV)
        if st["visible"] is not None:
            for i, w in enumerate(st["visible"][t:t + n].tolist()):
                hidden[i, p:] = torch.tensor([not (w >> b) & 1 for b in range(n)], device=DEV)
        o, e = torch.zeros((n, nq, hd), dtype=f64, device=DEV), torch.zeros((n, nq), dtype=f64, device=DEV)
        for h in range(nq):
            kh, vh = (y[:, h // G].reshape(-1, hd)[:total] for y in (k, v))
            z = (q[:, h] @ kh.t() / math.sqrt(hd)).masked_fill(hidden, -math.inf)
            e[:, h] = torch.logsumexp(z, -1)
            if c["op"] == "score":
                if h % G == 0:
                    scores[s, h // G, :total] = c["decay"] * st["score_in"][s, h // G, :total].to(f64)
                # normalisers given with the call are inputs
                scores[s, h // G, :total] += torch.exp(z - (st["lse"][t:t + n, h, None].to(f64) if c["lse"] else e[:, h, None])).sum(0)
            else:
                o[:, h] = torch.softmax(z, -1) @ vh
        outs.append(o.reshape(n, nq * hd))
        norms.append(e)
        t += n
    if c["op"] == "score":
        return {"score": scores}
    return {"out": torch.cat(outs), "lse": torch.cat(norms)} if c["lse"] else {"out": torch.cat(outs)}
