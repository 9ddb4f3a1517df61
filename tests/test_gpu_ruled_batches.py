"""Attention under a rule in batches of unlike sequences, and what its forms of many rows make of values that are not finite."""
import math

import pytest
import torch

from search_ops import seen

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def cache_ops():
    import cache_ops
    return cache_ops


def attend(c, q, out, rule, lse, scale=0.0):
    d = lambda k: torch.tensor(rule[k], dtype=torch.int32, device=DEV) if rule.get(k) is not None else None
    c.ctx.attend_ruled(0, c.lens, c.d_past, c.d_table, q, out, block=rule.get("block", 0), window=rule.get("window", 0), prefix=d("prefix"), first=d("first"),
                       end=d("end"), cap=rule.get("cap", 0.0), scale=scale, lse=lse)
    torch.cuda.synchronize()


def few(G, n):
    return n * G <= 32


# (heads, query heads of each, features, lens, past): two row tiles, 128 rows and 256 rows per workgroup for the longest ones
MIXED = [(2, 1, 64, [1, 20, 300, 32, 33], [200, 90, 100, 0, 500]), (2, 4, 128, [1, 8, 9, 40, 0, 3], [300, 41, 41, 500, 7, 64]),
         (16, 1, 128, [1, 2600, 32, 7], [900, 300, 64, 15]), (16, 8, 128, [3, 3500, 1, 4], [301, 300, 2000, 0]), (16, 8, 64, [2, 3600, 1], [700, 800, 33])]


@pytest.mark.parametrize("rule", [dict(block=1), dict(block=32, window=600), dict()])
@pytest.mark.parametrize("call", range(len(MIXED)))
def test_short_sequences_beside_long_ones(cache_ops, call, rule):
    """A sequence of at most 32 rows has its weights within 2^-15 and others within 2^-8, whatever else is in the call.  Queries and keys are
    small whole numbers, so that products are exact, and scores are off by the roundings of scale * log2(e) and of their shift alone."""
    nh, G, hd, lens, past = MIXED[call]
    c = cache_ops.Cache("bf16", nh, hd, lens, past, seed=call)
    g = torch.Generator().manual_seed(call)
    c.pool[:, :, 0] = torch.randint(-1, 2, c.pool[:, :, 0].shape, generator=g).to(torch.bfloat16).to(DEV)
    q = torch.randint(-1, 2, (c.T, nh * G * hd), generator=g).to(torch.bfloat16).to(DEV)
    out, lse = torch.full((c.T + 1, nh * G * hd), 3.0, dtype=torch.bfloat16, device=DEV), torch.zeros(c.T, nh * G, device=DEV)
    scale, pool, t0 = 0.25, c.pool.cpu(), 0
    attend(c, q, out, rule, lse, scale)
    assert (out[c.T:] == 3).all()
    for s, (n, p) in enumerate(zip(lens, past)):
        k, v = c.rows(s, p + n, pool)
        for i in range(n) if few(G, n) else sorted({0, 1, n // 3, n // 2, n - 2, n - 1}):
            ok = seen(rule, s, t0 + i, p + i, p + n)
            qi = q[t0 + i].cpu().double().view(-1, hd)
            for h in sorted({0, 1, nh * G - 1}):
                z = (k[:, h // G] @ qi[h] * scale)[ok]
                e = 2 * float(z.abs().max()) * 2.0 ** -22 + 2.0 ** -19
                w = torch.softmax(z, 0)
                ref, mag = w @ v[ok, h // G], w @ v[ok, h // G].abs()
                got = out[t0 + i].cpu().double().view(-1, hd)[h]
                bar = 2.0 ** -8 * ref.abs() + ((2.0 ** -15 if few(G, n) else 2.0 ** -8) + e) * mag
                assert ((got - ref).abs() <= bar).all(), (s, i, h, float(((got - ref).abs() / bar).max()))
                assert abs(float(lse[t0 + i, h]) - float(torch.logsumexp(z, 0))) <= e + 2.0 ** -21 * abs(float(torch.logsumexp(z, 0)))
        t0 += n
    c.close()


MANY = [(16, 1, 128, 2700, 300), (16, 2, 64, 2700, 300), (16, 8, 128, 3500, 300), (16, 16, 64, 3500, 301)]      # 128 and 256 rows per workgroup


@pytest.mark.parametrize("rule_name", ["causal", "block7", "prefix_block", "prefix_window", "documents"])
@pytest.mark.parametrize("call", range(len(MANY)))
def test_odd_values_among_many_rows(cache_ops, call, rule_name):
    """NaN and both infinities in a few features of some values, NaN in some keys: they reach the rows that see them, in those features, and
    nothing else; rows at the borders of groups and the last ones, all other features, against the definition."""
    nh, G, hd, n, p = MANY[call]
    c = cache_ops.Cache("bf16", nh, hd, [n], [p], seed=call, room=1000)
    size, total = 613, n + p
    at = torch.arange(p, total)
    rule = dict(causal=dict(block=1), block7=dict(block=7, cap=5.0), prefix_block=dict(block=32, prefix=[1000]),
                prefix_window=dict(window=700, prefix=[45], cap=30.0),
                documents=dict(first=(at // size * size).tolist(), end=(at // size * size + size).tolist()))[rule_name]
    odd, feature = [math.nan, math.inf, -math.inf], torch.arange(hd)
    places = [7, 60, p - 1, p, p + n // 4, p + n // 2 + 3, p + n // 2 + 40, total - 900, total - 1]
    for i, at in enumerate(places):
        c.set_rows(0, [at], v=torch.where(feature % 16 == i, odd[i % 3], 1.0).expand(1, nh, hd))
    # a key that some rows see: the first ones where there are windows and documents, else the last ones
    c.set_rows(0, [60 if rule_name in ("prefix_window", "documents") else total - 1], k=torch.full((1, nh, hd), math.nan))
    q, lse = c.randn(n, nh * G * hd, scale=1.5), torch.zeros(n, nh * G, device=DEV)
    out = torch.full((n + 1, nh * G * hd), 3.0, dtype=torch.bfloat16, device=DEV)
    attend(c, q, out, rule, lse)
    assert (out[n:] == 3).all()
    k, v = c.rows(0, total)
    rows = [0, 1, 126, 127, 128, 129, 255, 256, 257, 1023, 1024, n * G // 2, n * G // 2 + 1, n * G - 300, n * G - 257, n * G - 70, n * G - 2, n * G - 1]
    finite = 0
    for r in rows:
        i = r // G
        ok = seen(rule, 0, i, p + i, total)
        for head in (0, nh - 1):
            h = head * G + r % G
            qi = q[i].cpu().double().view(-1, hd)[h]
            z, size = k[:, head] @ qi / math.sqrt(hd), (k[:, head].abs() @ qi.abs() / math.sqrt(hd))[ok]
            e = float(size.nan_to_num(0.0).max()) * (hd + 4) * 2.0 ** -24 + rule.get("cap", 0.0) * 2.0 ** -21
            if rule.get("cap"):
                z = rule["cap"] * torch.tanh(z / rule["cap"])
            w = torch.softmax(z[ok], 0)
            # value by value: a weight of 0 is none, and only what is seen takes part
            ref, mag = w @ v[ok, head], w @ v[ok, head].abs()
            got, e = out[i].cpu().double().view(-1, hd)[h], 2 * e + 2.0 ** -19
            # float32 holds no weight below 2^-126 of the row's largest: it is 0, and 0 times a value that is not finite is no number
            lost = ((w / w.max() < 2.0 ** -126)[:, None] & ~v[ok, head].isfinite()).any(0)
            bar = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + e) * mag
            good = ((got - ref).abs() <= bar) | (got == ref) | (got.isnan() & ref.isnan()) | lost
            assert good.all(), (r, h, (~good).nonzero()[:4].tolist(), got[~good][:4], ref[~good][:4])
            finite += int(ref.isfinite().sum())
            norm, had = float(torch.logsumexp(z[ok], 0)), float(lse[i, h])
            assert math.isnan(norm) and math.isnan(had) or abs(had - norm) <= e + 2.0 ** -21 * abs(norm), (r, h)
    assert finite > len(rows) * hd // 3      # (of twice that many)
    c.close()


def test_two_launches_in_a_graph(cache_ops):
    """Short sequences beside one of many rows, captured and replayed between eager calls on other queries: the eager result, bit for bit."""
    c = cache_ops.Cache("bf16", 16, 128, [1, 2600, 7], [900, 300, 64], seed=6)
    q, s, graph = c.randn(c.T, 2048), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    out, ref = (torch.zeros(c.T, 2048, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    run = lambda o: c.ctx.attend_ruled(0, c.lens, c.d_past, c.d_table, q, o, block=1)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(out)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            run(out)
    torch.cuda.synchronize()
    for turn in range(4):
        q.copy_(c.randn(c.T, 2048))
        run(ref)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and out.abs().max() > 0, turn
    c.close()
