"""Attention of new tokens under a rule against its definition in 64 bits."""
import ctypes
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def m():
    import cache_ops
    import search_ops
    return cache_ops, search_ops


def attend(c, q, out, rule, lse=None, scale=0.0, lens=None, d_past=0):
    d = lambda k: torch.tensor(rule[k], dtype=torch.int32, device=DEV) if rule.get(k) is not None else None
    slope = torch.tensor(rule["slope"], dtype=torch.float32, device=DEV) if rule.get("slope") is not None else None
    c.ctx.attend_ruled(0, c.lens if lens is None else lens, c.d_past if d_past == 0 else d_past, c.d_table, q, out, block=rule.get("block", 0), window=rule.get("window", 0),
                       prefix=d("prefix"), first=d("first"), end=d("end"), cap=rule.get("cap", 0.0), slope=slope, scale=scale, lse=lse)
    torch.cuda.synchronize()


def documents(lens, past, size, both=True):
    at = [p + i for l, p in zip(lens, past) for i in range(l)]
    first = [a // size * size for a in at]
    return dict(first=first, end=[f + size for f in first] if both else None)


def slopes(n):
    return [2.0 ** (-8.0 * (i + 1) / n) for i in range(n)]


SHAPES = [
    # dtype, heads, head_dim, group, lens, past
    ("f32", 4, 64, 1, [5, 33, 1, 0, 17], [64, 0, 901, 40, 300]),
    ("bf16", 4, 64, 1, [5, 33, 1, 0, 17], [64, 0, 901, 40, 300]),
    ("bf16", 2, 128, 4, [70, 1, 19], [333, 1500, 0]),
    ("bf16", 3, 64, 3, [129, 64], [0, 77]),
    ("f32", 2, 128, 2, [40, 7], [50, 601]),
    ("bf16", 1, 128, 1, [1], [0]),
    ("bf16", 1, 64, 8, [300, 260], [0, 90]),
    ("bf16", 2, 128, 2, [333, 1], [50, 2]),
]
RULES = ["none", "causal", "block7", "window", "prefix_block", "prefix_window", "documents", "all", "empty"]


def make_rule(name, lens, past, nq):
    total = [l + p for l, p in zip(lens, past)]
    if name == "none":
        return {}
    if name == "causal":
        return dict(block=1)
    if name == "block7":
        return dict(block=7, cap=5.0)
    if name == "window":
        return dict(block=1, window=37, slope=slopes(nq))
    if name == "prefix_block":
        return dict(block=32, prefix=[max(0, n // 3) for n in total])
    if name == "prefix_window":
        return dict(window=20, prefix=[min(n, 19) for n in total], cap=30.0)
    if name == "documents":
        return dict(**documents(lens, past, 29), slope=slopes(nq))
    if name == "all":
        return dict(block=4, window=50, prefix=[min(n, 45) for n in total], **documents(lens, past, 61), cap=8.0, slope=[(-1) ** i * s for i, s in enumerate(slopes(nq))])
    # every third token sees nothing, the others end early
    T = sum(lens)
    return dict(block=1, first=[10 ** 6 if i % 3 == 0 else 0 for i in range(T)], end=[-5 if i % 3 == 1 else 12 for i in range(T)])


@pytest.mark.parametrize("rule_name", RULES)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_the_definition(m, shape, rule_name):
    cache, ops = m
    dtype, nh, hd, G, lens, past = SHAPES[shape]
    c = cache.Cache(dtype, nh, hd, lens, past, seed=shape)
    rule = make_rule(rule_name, lens, past, nh * G)
    q, out = c.randn(c.T, nh * G * hd, scale=1.5), torch.full((c.T + 2, nh * G * hd), 7.0, dtype=cache.TYPE[dtype], device=DEV)
    lse = torch.full((c.T + 2, nh * G), 7.0, device=DEV)
    attend(c, q, out, rule, lse)
    ops.check_attention(c, q, G, rule, out, lse)
    assert (out[c.T:] == 7).all() and (lse[c.T:] == 7).all()
    c.close()


@pytest.mark.parametrize("rule_name", ["none", "causal", "block7", "prefix_block", "prefix_window", "documents", "all"])
@pytest.mark.parametrize("dtype,nh,hd,G,lens,past", [("bf16", 2, 128, 1, [700], [0]), ("bf16", 1, 128, 3, [512, 100], [1500, 10]),
                                                     ("bf16", 2, 64, 2, [450, 900], [31, 0]), ("f32", 1, 64, 1, [260], [1000])])
def test_long_chunks(m, dtype, nh, hd, G, lens, past, rule_name):
    cache, ops = m
    c = cache.Cache(dtype, nh, hd, lens, past, seed=77)
    rule = make_rule(rule_name, lens, past, nh * G)
    if "first" in rule:
        rule.update(documents(lens, past, 313))
    if rule.get("window"):
        rule["window"] = 333
    q, out, lse = c.randn(c.T, nh * G * hd, scale=1.5), torch.zeros(c.T, nh * G * hd, dtype=cache.TYPE[dtype], device=DEV), torch.zeros(c.T, nh * G, device=DEV)
    attend(c, q, out, rule, lse)
    ops.check_attention(c, q, G, rule, out, lse)
    c.close()


def test_random_rules(m):
    """Rules of every kind at once, drawn; first and end of single tokens anywhere."""
    import random
    cache, ops = m
    rng = random.Random(5)
    for turn in range(24):
        dtype, nh, hd, G = rng.choice([("bf16", 2, 64, 1), ("bf16", 1, 128, 2), ("f32", 2, 64, 2), ("bf16", 1, 64, 5)])
        ns = rng.randint(1, 4)
        lens, past = [rng.choice([0, 1, 2, 16, 31, 90, 200]) for _ in range(ns)], [rng.choice([0, 1, 15, 16, 100, 500]) for _ in range(ns)]
        if sum(lens) == 0:
            lens[0] = 3
        T, total = sum(lens), [l + p for l, p in zip(lens, past)]
        rule = dict(block=rng.choice([0, 1, 3, 16, 64, 2 ** 31 - 1]), window=rng.choice([0, 1, 2, 33, 100, 2 ** 31 - 1]), cap=rng.choice([0.0, 3.0]),
                    prefix=rng.choice([None, [rng.choice([-3, 0, 1, 40, 10 ** 6]) for _ in range(ns)]]), slope=rng.choice([None, slopes(nh * G)]))
        if rule["prefix"]:      # (the definition takes positions that exist)
            given, rule["prefix"] = rule["prefix"], [min(max(p, 0), n) for p, n in zip(rule["prefix"], total)]
        if rng.random() < 0.5:
            rule["first"] = [rng.randint(-4, 60) for _ in range(T)]
        if rng.random() < 0.5:
            rule["end"] = [rng.randint(-4, 400) for _ in range(T)]
        c = cache.Cache(dtype, nh, hd, lens, past, seed=turn)
        q, out, lse = c.randn(T, nh * G * hd, scale=2.0), torch.zeros(T, nh * G * hd, dtype=cache.TYPE[dtype], device=DEV), torch.zeros(T, nh * G, device=DEV)
        attend(c, q, out, dict(rule, prefix=given) if rule["prefix"] else rule, lse)
        try:
            ops.check_attention(c, q, G, rule, out, lse)
        except AssertionError as e:
            raise AssertionError((turn, dtype, nh, hd, G, lens, past, {k: v for k, v in rule.items() if k not in ("first", "end")})) from e
        c.close()


@pytest.mark.parametrize("dtype,nh,hd,G,lens,past", [("bf16", 2, 64, 1, [40, 9], [70, 33]), ("f32", 1, 64, 2, [40], [70]), ("bf16", 1, 128, 2, [300], [40])])
def test_what_a_token_does_not_see_does_not_reach_it(m, dtype, nh, hd, G, lens, past):
    """NaN and infinities in keys and values outside of a row's window, document and order; the rows that see them get them."""
    cache, ops = m
    c = cache.Cache(dtype, nh, hd, lens, past, seed=9)
    odd = [math.nan, math.inf, -math.inf]
    total = lens[0] + past[0]
    at = [3, 20, 21, 64, past[0] - 1, past[0], past[0] + 7, total - 1]
    for i, p in enumerate(at):
        c.set_rows(0, [p], v=torch.full((1, nh, hd), 1.0) * torch.where(torch.arange(hd) % 5 == i % 5, odd[i % 3], 1.0))
    c.set_rows(0, [at[1], at[6]], k=torch.full((2, nh, hd), math.nan))
    rule = dict(block=1, window=25, prefix=[3] + [0] * (len(lens) - 1))
    q, out, lse = c.randn(c.T, nh * G * hd), torch.zeros(c.T, nh * G * hd, dtype=cache.TYPE[dtype], device=DEV), torch.zeros(c.T, nh * G, device=DEV)
    attend(c, q, out, rule, lse)
    clean = [i for i in range(lens[0]) if not any(ops.seen(rule, 0, i, past[0] + i, total)[p] for p in at)]
    hit = [i for i in range(lens[0]) if ops.seen(rule, 0, i, past[0] + i, total)[at[5]] and not any(ops.seen(rule, 0, i, past[0] + i, total)[at[k]] for k in (1, 6))]
    assert clean and hit
    ref = ops.attention(c, q, G, rule)[0]
    got = out.cpu().double().reshape(ref.shape)
    assert torch.isfinite(got[clean]).all() and torch.isfinite(lse.cpu()[clean]).all()
    assert (torch.isfinite(got[hit]) == torch.isfinite(ref[hit])).all()
    assert (torch.isnan(got[hit]) == torch.isnan(ref[hit])).all()
    # everything else as if nothing odd were there
    keep = torch.zeros(c.T, dtype=torch.bool)
    keep[clean] = True
    keep[lens[0]:] = True
    bar = (2.0 ** -6 if dtype == "bf16" else 2.0 ** -12)
    assert (got[keep] - ref[keep]).abs().max() <= bar * ref[keep].abs().max()
    c.close()


def test_strides_and_scale(m):
    cache, ops = m
    c = cache.Cache("bf16", 2, 64, [50, 3], [100, 7], seed=4)
    wide = c.randn(c.T, 5 * 128)
    q, out = wide[:, 128:256], torch.zeros(c.T, 3 * 128, dtype=torch.bfloat16, device=DEV)
    attend(c, q, out[:, 128:256], dict(block=1), scale=0.3)
    ops.check_attention(c, q.contiguous(), 1, dict(block=1), out[:, 128:256].contiguous(), scale=0.3)
    assert (out[:, :128] == 0).all() and (out[:, 256:] == 0).all()
    c.close()


def test_no_cached_positions_and_the_rule_of_attend(m):
    """Without a rule it is dinfer_attend; d_past null is no past."""
    cache, ops = m
    c = cache.Cache("bf16", 4, 64, [40, 3], [0, 0], seed=8)
    q, out, same = c.randn(c.T, 256), torch.zeros(c.T, 256, dtype=torch.bfloat16, device=DEV), torch.zeros(c.T, 256, dtype=torch.bfloat16, device=DEV)
    attend(c, q, out, {}, d_past=None)
    c.ctx.attend(0, c.lens, None, c.d_table, q, same)
    torch.cuda.synchronize()
    ops.check_attention(c, q, 1, {}, out)
    ops.check_attention(c, q, 1, {}, same)
    c.close()


@pytest.mark.parametrize("dtype,lens,past", [("bf16", [33, 1], [900, 1100]), ("bf16", [400], [300]), ("f32", [20], [700])])
def test_streams_and_graphs(m, dtype, lens, past):
    """Captured once, replayed between eager calls on other queries: every replay is the eager result, bit for bit."""
    cache, ops = m
    c = cache.Cache(dtype, 2, 64, lens, past, seed=2)
    q = c.randn(c.T, 128)
    out, ref = (torch.zeros(c.T, 128, dtype=cache.TYPE[dtype], device=DEV) for _ in range(2))
    lse = torch.zeros(c.T, 2, device=DEV)
    prefix = torch.tensor([5] * len(lens), dtype=torch.int32, device=DEV)
    run = lambda o: c.ctx.attend_ruled(0, c.lens, c.d_past, c.d_table, q, o, block=1, window=333, prefix=prefix, cap=9.0, lse=lse)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(out)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            run(out)
    torch.cuda.synchronize()
    for turn in range(4):
        q.copy_(c.randn(c.T, 128))
        run(ref)
        torch.cuda.synchronize()
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref), turn
        ops.check_attention(c, q, 1, dict(block=1, window=333, prefix=[5] * len(lens), cap=9.0), out, lse)
    c.close()


def test_refusals(m):
    cache, _ = m
    from paper_2510_08666_amd import binding as b
    c = cache.Cache("bf16", 2, 64, [3], [10], seed=1)
    q, out = c.randn(3, 128), torch.full((3, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    ok = dict(block=1)
    for bad in (dict(block=-1), dict(window=-1), dict(cap=-1.0), dict(cap=math.nan), dict(cap=1e-31), dict(cap=math.inf)):
        with pytest.raises(b.DinferError):
            attend(c, q, out, bad)
    with pytest.raises(b.DinferError):
        attend(c, q, out, ok, scale=-1.0)
    with pytest.raises(b.DinferError):
        attend(c, c.randn(500, 128), torch.zeros(500, 128, dtype=torch.bfloat16, device=DEV), ok, lens=[500])
    for bad in (dict(prefix=torch.zeros(1, device=DEV)), dict(first=torch.zeros(2, dtype=torch.int32, device=DEV)), dict(slope=torch.zeros(1, device=DEV)),
                dict(end=torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            c.ctx.attend_ruled(0, c.lens, c.d_past, c.d_table, q, out, **bad)
    assert b.lib.dinfer_attend_ruled(c.ctx.h, 0, 1, (ctypes.c_int32 * 1)(3), None, c.d_table.data_ptr(), c.d_table.shape[1], q.data_ptr(), 128, 2,
                                     None, 0.0, out.data_ptr(), 128, None, None) == -1
    torch.cuda.synchronize()
    assert (out == 5).all()
    c.close()


@pytest.mark.parametrize("dtype,nh,hd,G,lens,past,rule_name", [
    ("bf16", 16, 128, 1, [1100, 40, 0, 900], [300, 1500, 7, 0], "causal"), ("bf16", 8, 128, 4, [700, 333], [0, 1000], "block7"),
    ("bf16", 8, 64, 4, [1200, 900], [77, 500], "prefix_block"), ("bf16", 4, 128, 8, [600, 500], [900, 0], "all"),
    ("bf16", 16, 128, 1, [2000, 1900], [0, 31], "documents"), ("bf16", 16, 128, 2, [800], [100], "prefix_window"),
    ("bf16", 16, 128, 8, [3500], [300], "causal"), ("bf16", 16, 128, 8, [3600, 5], [300, 0], "documents"), ("bf16", 16, 128, 16, [3700], [300], "documents"), ("bf16", 16, 64, 16, [3500], [301], "prefix_block"),
    ("bf16", 16, 128, 8, [3500], [300], "prefix_window"), ("bf16", 16, 128, 8, [1800, 1700], [0, 300], "all")])
def test_the_form_of_many_rows(m, dtype, nh, hd, G, lens, past, rule_name):
    """Calls that are large enough for it: a few tokens of them against the definition."""
    cache, ops = m
    c = cache.Cache(dtype, nh, hd, lens, past, seed=5, room=2000)
    rule = make_rule(rule_name, lens, past, nh * G)
    if "first" in rule:
        rule.update(documents(lens, past, 613))
    if rule.get("window"):
        rule["window"] = 700
    q, out, lse = c.randn(c.T, nh * G * hd, scale=1.5), torch.full((c.T + 1, nh * G * hd), 3.0, dtype=cache.TYPE[dtype], device=DEV), torch.zeros(c.T, nh * G, device=DEV)
    odd = past[0] + lens[0] // 2
    c.set_rows(0, [odd], v=torch.full((1, nh, hd), math.inf))
    attend(c, q, out, rule, lse)
    assert (out[c.T:] == 3).all()
    # a sequence of the chosen tokens only: each a sequence of its own behind the same pages
    t0 = 0
    for s, (n, p) in enumerate(zip(lens, past)):
        for i in sorted({0, 1, n // 3, n // 2, n // 2 + 1, n - 31, n - 1}):
            if not 0 <= i < n:
                continue
            ok = ops.seen(rule, s, t0 + i, p + i, p + n)
            k, v = c.rows(s, p + n)
            at = torch.arange(p + n)
            for h in (0, nh * G - 1):
                z = k[:, h // G] @ q[t0 + i].cpu().double().view(-1, hd)[h] / math.sqrt(hd)
                size = k[:, h // G].abs() @ q[t0 + i].cpu().double().view(-1, hd)[h].abs() / math.sqrt(hd)
                e = float(size.max()) * (hd + 4) * 2.0 ** -24 + rule.get("cap", 0.0) * 2.0 ** -21
                if rule.get("cap"):
                    z = rule["cap"] * torch.tanh(z / rule["cap"])
                if rule.get("slope") is not None:
                    z = z - rule["slope"][h] * (at - p - i).abs()
                    e += abs(rule["slope"][h]) * (p + n) * 2.0 ** -22
                w = torch.softmax(z[ok], 0)
                ref, mag = w @ v[ok, h // G], w @ v[ok, h // G].abs()
                got = out[t0 + i].cpu().double().view(-1, hd)[h]
                e = 2 * e + 2.0 ** -19
                bar = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + e) * mag
                # float32 holds no weight below 2^-126 of the row's largest: it is 0, and 0 times a value that is not finite is no number
                lost = ((w / w.max() < 2.0 ** -126)[:, None] & ~v[ok, h // G].isfinite()).any(0)
                assert (((got - ref).abs() <= bar) | (got == ref) | lost).all(), (s, i, h, float((got - ref).abs().max()))
                norm = float(torch.logsumexp(z[ok], 0))
                assert abs(float(lse[t0 + i, h]) - norm) <= e + 2.0 ** -21 * abs(norm)
        t0 += n
    c.close()


@pytest.mark.parametrize("lens,past,G", [([3, 40], [500, 0], 1), ([1300], [700], 1), ([4000], [300], 1), ([3500], [300], 8)])
def test_pages_beyond_32_bits(m, lens, past, G):
    """The same rows in pages whose elements are numbered from 2^32 on (a pool of 8 GiB and more): the same bits, in every form."""
    from paper_2510_08666_amd import binding
    cache, ops = m
    c = cache.Cache("bf16", 16, 128, lens, past, seed=3)
    first = 2 ** 32 // (2 * 16 * 128 * 16)      # elements of a page
    far = binding.Context(c.cfg, first + c.n_pages, c.ns, 64, c.max_pos)
    far.kv.view(torch.bfloat16).view(first + c.n_pages, -1)[first:].copy_(c.pool.view(c.n_pages, -1))
    far.kv.view(torch.bfloat16).view(first + c.n_pages, -1)[:c.n_pages].zero_()
    q = c.randn(c.T, G * 2048)
    outs = [torch.zeros(c.T, G * 2048, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for ctx, table, out in ((c.ctx, c.d_table, outs[0]), (far, torch.where(c.d_table >= 0, c.d_table + first, c.d_table), outs[1])):
        ctx.attend_ruled(0, c.lens, c.d_past, table, q, out, block=1)
    torch.cuda.synchronize()
    assert torch.equal(*outs) and outs[0].abs().max() > 0
    far.close()
    c.close()
