"""The paged cache's operators against float64: append (norms, rotation, page layout), attention under visibility words,
gathered attention weight, eviction; runs of them together; streams, graphs and refusals."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 4, 128), ("bf16", 3, 64), ("f32", 2, 128), ("f32", 5, 64)]


@pytest.fixture(scope="module")
def m():
    import cache_ops
    return cache_ops


# ------------------------------------------------------------------------------------------------ append

def turned(x, pos, dim, interleaved, f, size):
    """Rotation in float64 of x [T][heads][features]."""
    import torch
    y = x.clone()
    ang = pos.double()[:, None] * f
    c, s = (ang.cos() * size)[:, None], (ang.sin() * size)[:, None]
    ia, ib = (slice(0, dim, 2), slice(1, dim, 2)) if interleaved else (slice(0, dim // 2), slice(dim // 2, dim))
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


def frequencies(r, theta, scaling, factor, original):
    import torch
    j = torch.arange(r // 2, dtype=torch.float64)
    if scaling == "ntk":
        theta = theta * factor ** (r / (r - 2))
    f = theta ** (-2 * j / r)
    if scaling == "linear":
        f = f / factor
    if scaling == "yarn":
        c = [r * math.log(original / (b * 2 * math.pi)) / (2 * math.log(theta)) for b in (32, 1)]
        lo, hi = max(0, math.floor(c[0])), min(r - 1, math.ceil(c[1]))
        ramp = ((j - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1
    return f, 1.0


APPENDS = [([1, 0, 33, 64, 7, 16], [0, 5, 16, 500, 31, 48]), ([1], [0]), ([1], [1000]), ([17], [15]), ([300, 5], [0, 3])]


@pytest.mark.parametrize("dtype,heads,hd", SHAPES)
@pytest.mark.parametrize("i", range(len(APPENDS)))
@pytest.mark.parametrize("dim,interleaved,scaling,norm,group,custom", [
    (0, False, "plain", False, 1, False), (1, False, "plain", True, 2, True), (1, True, "yarn", True, 1, True), (2, False, "ntk", False, 3, True),
    (4, True, "linear", True, 1, False), (20, False, "plain", True, 2, True), (20, True, "yarn", False, 1, True), (2, False, "linear", True, 8, False)])
def test_append(m, dtype, heads, hd, i, dim, interleaved, scaling, norm, group, custom):
    torch = m.torch
    lens, past = APPENDS[i]
    c = m.Cache(dtype, heads, hd, lens, past, seed=i)
    T, nq = c.T, heads * group
    qkv = c.randn(T, (nq + 2 * heads) * hd, scale=2.0)
    q, k, v = qkv.split([nq * hd, heads * hd, heads * hd], 1)
    pad = c.randn(T + 3, nq * hd + 32)                          # queries go into part of a wider matrix
    before, pool0 = pad.clone(), c.pool.cpu().clone()
    gains = [(1 + 0.2 * torch.randn(hd, generator=c.g)).to(m.DEV) for _ in range(2)] if norm else [None, None]
    at = torch.cat([torch.arange(p, p + l) for l, p in zip(lens, past)])
    pos = torch.randint(0, 3000, (T,), generator=c.g, dtype=torch.int32) if custom else None
    r = hd if dim in (0, 1) else dim if dim == 20 else hd // dim
    kw = {}
    if dim:
        rot = m.binding.rotary(r, interleaved, 5000.0, scaling, 1.0 if scaling == "plain" else 4.0, 2048)
        kw = dict(rotary=rot, rotary_table=m.binding.rotary_table(rot, 3000))
    c.ctx.kv_append(0, lens, c.d_past, c.d_table, q, k, v, pad[:T, 16:16 + nq * hd], q_gain=gains[0], k_gain=gains[1], eps=1e-5,
                    positions=None if pos is None else pos.to(m.DEV), **kw)
    torch.cuda.synchronize()
    f, size = frequencies(r, 5000.0 if dim else 10000.0, scaling, 4.0, 2048) if dim else frequencies(hd, 10000.0, "plain", 1, 1)
    where = at if pos is None else pos
    half, e32 = m.HALF_STEP[dtype], 2.0 ** -24

    def normed(x, gain):
        x = x.cpu().double().reshape(T, -1, hd)
        return x if gain is None else x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * gain.cpu().double()

    def check(got, x, what):
        ref = turned(x, where, r, interleaved, f, size)
        mag = turned(x.abs(), torch.zeros(T), r, interleaved, f, size).abs()
        a = turned(x.abs(), torch.full((T,), 1.0), r, interleaved, f * 0 + math.pi / 2, size).abs()
        # a norm's sum of hd squares (relative hd/2 steps of 2^-24 on its root at most), two products and a sum: float32; one rounding
        bar = half * ref.abs() + ((hd / 2 + 8) * e32) * (mag + a) + 1e-30
        bad = ~((got - ref).abs() <= bar)
        assert not bad.any(), (what, bad.nonzero()[:4], got[bad][:4], ref[bad][:4])

    check(pad[:T, 16:16 + nq * hd].cpu().double().reshape(T, nq, hd), normed(q, gains[0]), "q")
    pad[:T, 16:16 + nq * hd] = before[:T, 16:16 + nq * hd]
    assert torch.equal(pad, before)
    pool = c.pool.cpu()
    kk = torch.cat([c.rows(s, l + p, pool)[0][p:] for s, (l, p) in enumerate(zip(lens, past))])
    vv = torch.cat([c.rows(s, l + p, pool)[1][p:] for s, (l, p) in enumerate(zip(lens, past))])
    check(kk, normed(k, gains[1]), "k")
    assert torch.equal(vv, v.cpu().double().reshape(T, heads, hd))
    # every other row of the pool is as it was
    keep = torch.ones(c.n_pages, m.PAGE, dtype=torch.bool)
    for s, (l, p) in enumerate(zip(lens, past)):
        for x in range(p, p + l):
            keep[int(c.table[s, x // m.PAGE]), x % m.PAGE] = False
    for a, b in zip(c.views(pool), c.views(pool0)):
        assert torch.equal(a.movedim(3, 1)[keep], b.movedim(3, 1)[keep])
    c.close()


def test_append_keys_and_values_only_and_in_place(m):
    torch = m.torch
    c = m.Cache("bf16", 4, 128, [19, 2], [7, 100], seed=3)
    q, k, v = c.randn(c.T, 512), c.randn(c.T, 512), c.randn(c.T, 512)
    want = torch.empty_like(q)
    c.ctx.kv_append(0, c.lens, c.d_past, c.d_table, q, k, v, want)
    pool = c.pool.clone()
    c.pool.zero_()
    c.ctx.kv_append(0, c.lens, c.d_past, c.d_table, None, k, v, None)
    rows = [c.rows(s, l + p) for s, (l, p) in enumerate(zip(c.lens, c.past))]
    ref = [c.rows(s, l + p, pool.cpu()) for s, (l, p) in enumerate(zip(c.lens, c.past))]
    for s in range(2):
        for a, b in zip(rows[s], ref[s]):
            assert torch.equal(a[c.past[s]:], b[c.past[s]:]) and not a[:c.past[s]].any()
    c.ctx.kv_append(0, c.lens, c.d_past, c.d_table, q, k, v, q)
    assert torch.equal(q, want)
    c.close()


def test_append_like_the_step(m):
    """The context's own rotation: the same tables as the step's projection, element for element within a rounding."""
    torch = m.torch
    c = m.Cache("f32", 2, 64, [40], [9000], seed=1, max_pos=9100)
    k = c.randn(40, 128)
    c.ctx.kv_append(0, [40], c.d_past, c.d_table, None, k, k, None)
    got, _ = c.ctx.kv_read(0, c.d_table[0], 9000, 40)
    f, _ = frequencies(64, 10000.0, "plain", 1, 1)
    ref = turned(k.cpu().double().reshape(40, 2, 64), torch.arange(9000, 9040), 64, False, f, 1.0)
    assert (got.cpu().double().reshape(40, 2, 64) - ref).abs().max() <= 4 * 2.0 ** -24 * 2 * float(k.abs().max())
    c.close()


# ------------------------------------------------------------------------------------------------ attend

# (past 4001 and more: keys cut into parts; many sequences: the longest parts first)
LENS = [([1, 0, 33, 64, 7], [0, 5, 16, 500, 31]), ([1], [0]), ([1], [2000]), ([64], [8000]), ([2, 5, 31], [0, 0, 1]),
        ([20, 32, 1, 3, 64, 40], [800, 31, 1600, 0, 4001, 768]), ([3, 0, 7, 64] * 12, [40 * i for i in range(48)])]


def attend_case(m, dtype, heads, hd, i, kind, group, columns=0):
    torch = m.torch
    lens, past = LENS[i]
    c = m.Cache(dtype, heads, hd, lens, past, seed=10 + i, columns=columns)
    q = c.randn(c.T, heads * group * hd + 16, scale=1.5)[:, :heads * group * hd]
    words = None
    if kind == "tree":
        words = m.tree_words(c.g, lens)
    elif kind == "causal":
        words = [(2 << j) - 1 for l in lens for j in range(l)]
    elif kind == "empty":       # every second token sees no new one: with nothing cached, nothing at all
        words = [0 if j % 2 else (1 << 63) | 5 for l in lens for j in range(l)]
    wide = c.randn(c.T + 1, heads * group * hd + 32)
    before = wide.clone()
    out = wide[:c.T, 16:16 + heads * group * hd]
    lse = torch.full((c.T + 1, heads * group), 7.0, device=m.DEV)
    c.ctx.attend(0, lens, c.d_past, c.d_table, q, out, visible=None if words is None else m.word_tensor(words), lse=lse[:c.T],
                 scale=0.0 if i % 2 else 0.11)
    torch.cuda.synchronize()
    m.check_attention(c, q, group, out, lse[:c.T], words, None if i % 2 else 0.11)
    assert (lse[c.T] == 7).all()
    first = out.clone()
    wide[:c.T, 16:16 + heads * group * hd] = before[:c.T, 16:16 + heads * group * hd]
    assert torch.equal(wide, before)
    c.ctx.attend(0, lens, c.d_past, c.d_table, q, out, visible=None if words is None else m.word_tensor(words), scale=0.0 if i % 2 else 0.11)
    assert torch.equal(first, out)          # the same bits, with or without normalisers
    c.close()


@pytest.mark.parametrize("dtype,heads,hd", SHAPES)
@pytest.mark.parametrize("i", range(len(LENS)))
@pytest.mark.parametrize("kind,group", [("none", 1), ("tree", 1), ("tree", 3), ("causal", 8), ("empty", 2)])
def test_attend(m, dtype, heads, hd, i, kind, group):
    attend_case(m, dtype, heads, hd, i, kind, group)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("i,kind,group", [(0, "tree", 3), (3, "causal", 8), (4, "empty", 9), (5, "tree", 5)])
def test_attend_much_work(m, hd, i, kind, group):
    """Many cache heads and page-table rows of 32768 positions: what a call has to do at most chooses the form of many rows."""
    attend_case(m, "bf16", 20, hd, i, kind, group, columns=2048)


@pytest.mark.parametrize("columns", [0, 2048])
def test_attend_long_runs_without_words(m, columns):
    torch = m.torch
    heads = 8 if columns else 2
    c = m.Cache("bf16", heads, 64, [300, 65], [70, 0], seed=5, columns=columns)
    q = c.randn(c.T, heads * 2 * 64)
    out, lse = torch.empty_like(q), torch.empty(c.T, heads * 2, device=m.DEV)
    c.ctx.attend(0, c.lens, c.d_past, c.d_table, q, out, lse=lse)
    m.check_attention(c, q, 2, out, lse)
    c.close()


def hidden_case(m, dtype, heads, hd, past, group, columns=0):
    torch = m.torch
    n = 30
    c = m.Cache(dtype, heads, hd, [n, 9], [past, 3], seed=7, columns=columns)
    bad = [3, 11, 12, 29]
    kv = torch.randn(4, heads, hd, generator=c.g)
    kv[0], kv[1, :, ::3], kv[2, :, 1::2], kv[3] = math.nan, math.inf, -math.inf, math.nan
    c.set_rows(0, [past + b for b in bad], k=torch.where(torch.isnan(kv), kv, torch.full_like(kv, math.nan)), v=kv)
    behind = [x for x in range(past + n, -(-(past + n) // m.PAGE) * m.PAGE)]
    junk = torch.full((len(behind), heads, hd), math.nan)
    c.set_rows(0, behind, k=junk, v=junk)
    words = m.tree_words(c.g, [n, 9])
    hide = ~sum(1 << b for b in bad)
    words = [w & hide if t < n else w for t, w in enumerate(words)]
    nq = heads * group
    q = c.randn(c.T, nq * hd)
    out, lse = torch.empty_like(q), torch.empty(c.T, nq, device=m.DEV)

    def run(words):
        c.ctx.attend(0, c.lens, c.d_past, c.d_table, q, out, visible=m.word_tensor(words), lse=lse)
        torch.cuda.synchronize()
        m.check_attention(c, q, group, out, lse, words)

    run(words)
    assert torch.isfinite(out).all()
    # values alone: the keys are fine, tokens 0 .. 4 see the infinite value
    c.set_rows(0, [past + b for b in bad], k=torch.randn(4, heads, hd, generator=c.g))
    words = [w | (1 << 11) if t < 5 else w for t, w in enumerate(words)]
    run(words)
    o = out[:5].view(5, nq, hd)
    assert torch.isinf(o[..., ::3]).all() and torch.isfinite(o[..., 1::3]).all() and torch.isfinite(out[5:]).all()
    # tokens 5 and 6 see both infinities (NaN where they meet), token 7 the NaN
    words = [w | (1 << 11) | (1 << 12) if t in (5, 6) else w | (1 << 29) if t == 7 else w for t, w in enumerate(words)]
    run(words)
    assert torch.isnan(out[7]).all() and torch.isnan(out[5].view(nq, hd)[:, 3::6]).all() and torch.isfinite(out[8:]).all()
    # a key that is not a number, where it is seen
    c.set_rows(0, [past + 12], k=torch.full((1, heads, hd), math.nan))
    words = [w | (1 << 12) if t == 8 else w for t, w in enumerate(words)]
    c.ctx.attend(0, c.lens, c.d_past, c.d_table, q, out, visible=m.word_tensor(words), lse=lse)
    assert torch.isnan(out[8]).all() and torch.isnan(lse[8]).all() and torch.isfinite(out[9:]).all()
    c.close()


@pytest.mark.parametrize("dtype,heads,hd", SHAPES)
@pytest.mark.parametrize("past", [0, 37, 900])
@pytest.mark.parametrize("group", [1, 2, 3, 9])
def test_attend_what_is_hidden_does_not_reach(m, dtype, heads, hd, past, group):
    """NaN and infinities in new keys and values that a token does not see, and behind the last key; those it sees do reach it.
    (The groups choose the forms: 30, 60, 90 and 270 rows per cache head.)"""
    hidden_case(m, dtype, heads, hd, past, group)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("past", [0, 37, 900])
@pytest.mark.parametrize("group", [3, 9])
def test_attend_what_is_hidden_does_not_reach_much_work(m, hd, past, group):
    """The same in the form of many rows, of 90 rows and of 270."""
    hidden_case(m, "bf16", 20, hd, past, group, columns=2048)


def test_attend_extreme_scores(m):
    """Keys whose scores are far apart, in the type's highest and lowest values: the running maximum moves by thousands."""
    torch = m.torch
    c = m.Cache("bf16", 2, 64, [3], [200], seed=9)
    c.set_rows(0, [5, 70, 199, 201], k=torch.stack([300 * torch.ones(2, 64), -300 * torch.ones(2, 64), 1e4 * torch.ones(2, 64), torch.ones(2, 64)]))
    q = torch.ones(3, 128, device=m.DEV, dtype=torch.bfloat16) * torch.tensor([[1.0], [-1.0], [0.0]], device=m.DEV, dtype=torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(3, 2, device=m.DEV)
    c.ctx.attend(0, [3], c.d_past, c.d_table, q, out, lse=lse)
    m.check_attention(c, q, 1, out, lse)
    c.close()


# ------------------------------------------------------------------------------------------------ score

@pytest.mark.parametrize("dtype,heads,hd", SHAPES)
@pytest.mark.parametrize("i", range(len(LENS)))
@pytest.mark.parametrize("tree,group,given,decay", [(False, 1, False, 1.0), (True, 2, True, 0.5), (True, 8, False, 0.9)])
def test_score(m, dtype, heads, hd, i, tree, group, given, decay):
    torch = m.torch
    lens, past = LENS[i]
    c = m.Cache(dtype, heads, hd, lens, past, seed=20 + i)
    q = c.randn(c.T, heads * group * hd, scale=1.5)
    words = m.tree_words(c.g, lens) if tree else None
    if tree and lens[-1] > 2:
        words[-1] = 0                           # a token that sees no new one
    vis = None if words is None else m.word_tensor(words)
    width = max(l + p for l, p in zip(lens, past)) + 3
    old = torch.rand(c.ns, heads, width, generator=c.g).to(m.DEV)
    new = torch.full_like(old, -5.0)
    lse = None
    if given:
        lse, out = torch.empty(c.T, heads * group, device=m.DEV), torch.empty_like(q)
        c.ctx.attend(0, lens, c.d_past, c.d_table, q, out, visible=vis, lse=lse)
    c.ctx.kv_score(0, lens, c.d_past, c.d_table, q, new, score_in=old, decay=decay, visible=vis, lse=lse)
    torch.cuda.synchronize()
    _, _, weights, _, err = c.attention(q, group, words)
    got = new.cpu().double()
    for s in range(c.ns):
        n = lens[s] + past[s] if lens[s] else 0
        w = weights[s].reshape(lens[s], heads, group, -1).sum((0, 2)) if lens[s] else torch.zeros(heads, 0)
        ref = decay * old[s, :, :n].cpu().double() + w[:, :n]
        # a weight's relative error: twice a score's absolute one, exponential and normaliser 2^-19; a row's sum in 2^-24 steps
        bar = (2 * err + 2.0 ** -18) * w[:, :n] + 2.0 ** -22 * ref + 1e-30
        assert ((got[s, :, :n] - ref).abs() <= bar).all()
        assert (got[s, :, n:] == -5).all()
    again = old.clone()
    c.ctx.kv_score(0, lens, c.d_past, c.d_table, q, again, score_in=again, decay=decay, visible=vis, lse=lse)     # in place, the same bits
    for s in range(c.ns):
        n = lens[s] + past[s] if lens[s] else 0
        assert torch.equal(again[s, :, :n], new[s, :, :n])
    narrow = torch.full((c.ns, heads, 40), -5.0, device=m.DEV)              # positions behind the width are not scored
    c.ctx.kv_score(0, lens, c.d_past, c.d_table, q, narrow, visible=vis)
    for s in range(c.ns):
        n = min(40, lens[s] + past[s]) if lens[s] else 0
        w = weights[s].reshape(lens[s], heads, group, -1).sum((0, 2)) if lens[s] else torch.zeros(heads, 0)
        assert ((narrow[s, :, :n].cpu().double() - w[:, :n]).abs() <= (2 * err + 2.0 ** -18) * w[:, :n] + 1e-30).all()
        assert (narrow[s, :, n:] == -5).all()
    c.close()


def test_score_hidden_keys(m):
    torch = m.torch
    c = m.Cache("bf16", 2, 128, [12], [40], seed=31)
    c.set_rows(0, [45, 47], k=torch.stack([torch.full((2, 128), math.nan), torch.full((2, 128), math.inf)]))
    words = [w & ~((1 << 5) | (1 << 7)) for w in m.tree_words(c.g, [12])]
    q = c.randn(12, 256)
    new = torch.zeros(1, 2, 60, device=m.DEV)
    c.ctx.kv_score(0, [12], c.d_past, c.d_table, q, new, visible=m.word_tensor(words))
    assert torch.isfinite(new).all() and (new[0, :, [45, 47]] == 0).all()
    assert (new.sum(-1) - 12).abs().max() < 12 * 2.0 ** -16
    c.close()


# ------------------------------------------------------------------------------------------------ evict

def chosen(score, n, keep, sink, recent):
    """Positions kept, by the definition, from float32 scores."""
    x = np.where(np.isnan(score[:n]), -np.inf, score[:n]).astype(np.float64)
    nan = np.isnan(score[:n])
    order = sorted(range(n), key=lambda i: (0 if i < sink or i >= n - recent else 1, nan[i], -x[i], i))
    return sorted(order[:min(n, keep)])


@pytest.mark.parametrize("dtype,heads,hd", SHAPES)
@pytest.mark.parametrize("past,keep,sink,recent", [
    ([700, 3, 64, 0, 65], 64, 4, 16), ([1], 1, 0, 0), ([5000, 1025], 1024, 0, 0), ([4096, 17, 4095], 1000, 16, 984), ([33], 17, 0, 17),
    ([9000], 3001, 5, 1000)])
def test_evict(m, dtype, heads, hd, past, keep, sink, recent):
    torch = m.torch
    L, ns = 2, len(past)
    c = m.Cache(dtype, heads, hd, [0] * ns, past, layers=3, seed=40 + keep, spare=ns * (-(-keep // 16)) + 3)
    width = max(past) + 2
    score = torch.rand(L, ns, heads, width, generator=c.g)
    u = torch.rand(score.shape, generator=c.g)
    score = torch.where(u < 0.3, torch.zeros_like(score), torch.where(u < 0.6, (score * 4).round() / 4, score))
    score = torch.where((u > 0.97) & (u < 0.98), -score, score)
    score = torch.where((u > 0.98) & (u < 0.985), torch.full_like(score, math.nan), score)
    score = torch.where(u > 0.997, torch.full_like(score, math.inf), score)
    score = torch.where((u > 0.99) & (u < 0.993), torch.full_like(score, -math.inf), score)
    score = torch.where((u > 0.2) & (u < 0.3), -torch.zeros_like(score), score)
    P = -(-keep // 16)
    new_table = torch.full((ns, P + 1), -7, dtype=torch.int32)
    new_table[:, :P] = c.free[:ns * P].reshape(ns, P)
    pool0 = c.pool.cpu().clone()
    d_score = score.to(m.DEV)
    out = torch.full_like(d_score, 9.0)
    kept = torch.full((L, ns, heads, keep), 77, dtype=torch.int32, device=m.DEV)
    new_len = torch.full((ns + 1,), 5, dtype=torch.int32, device=m.DEV)
    c.ctx.kv_evict(1, L, keep, sink, recent, d_score, c.d_past, c.d_table, new_table.to(m.DEV), kept, new_len, score_out=out)
    torch.cuda.synchronize()
    assert new_len.tolist() == [min(p, keep) for p in past] + [5]
    pool, kept, out = c.pool.cpu(), kept.cpu(), out.cpu()
    touched = torch.zeros(3, c.n_pages, m.PAGE, dtype=torch.bool)
    for l in range(L):
        for s in range(ns):
            n = min(past[s], keep)
            old_k, old_v = c.rows(s, past[s], pool0, 1 + l)
            got_k, got_v = c.rows(s, n, pool, 1 + l, new_table)
            for x in range(n):
                touched[1 + l, int(new_table[s, x // 16]), x % 16] = True
            for h in range(heads):
                want = chosen(score[l, s, h].numpy(), past[s], keep, sink, recent)
                assert kept[l, s, h].tolist() == want + [-1] * (keep - n), (l, s, h)
                assert torch.equal(got_k[:, h], old_k[want, h]) and torch.equal(got_v[:, h], old_v[want, h])
                a, b = out[l, s, h, :n], score[l, s, h][want]
                assert ((a == b) | (a.isnan() & b.isnan())).all() and (out[l, s, h, n:] == 0).all()
    for l in range(3):
        for a, b in zip(c.views(pool, l), c.views(pool0, l)):
            assert torch.equal(a.movedim(3, 1)[~touched[l]], b.movedim(3, 1)[~touched[l]])
    c.close()
