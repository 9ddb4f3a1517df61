"""Capped scores: caps from below the scores' size to far above it, which change nothing."""
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


def definition(c, q, group, cap, slope, scale):
    """out, lse, sum of p |v|, and a bound on a score's error that follows the scores and not the cap: (hd + 4) roundings of the product's
    size, 2^-20 of the score for the cap (2^-21.1 at most: for tanh next to 1/2, where the exponential, the reciprocal and two sums lose a step each
    of a number below 1; two products and the scale, half a step each), three roundings of the bias."""
    pool, nq, t, err = c.pool.cpu(), c.nh * group, 0, 0.0
    q = q.cpu().double().reshape(c.T, nq, c.hd)
    out, lse, mag = torch.zeros(c.T, nq, c.hd).double(), torch.zeros(c.T, nq).double(), torch.zeros(c.T, nq, c.hd).double()
    for s in range(c.ns):
        n, p = c.lens[s], c.past[s]
        k, v = c.rows(s, n + p, pool)
        ok = torch.stack([seen(dict(block=1), s, t + i, p + i, n + p) for i in range(n)])
        away = (torch.arange(n + p)[None] - torch.arange(p, p + n)[:, None]).abs().double()
        for h in range(nq):
            z = q[t:t + n, h] @ k[:, h // group].t() * scale
            err = max(err, float((q[t:t + n, h].abs() @ k[:, h // group].abs().t() * scale).max()) * (c.hd + 4) * 2.0 ** -24)
            if cap:
                z = cap * torch.tanh(z / cap)
                err = max(err, float(z.abs().max()) * 2.0 ** -20)
            if slope is not None:
                z = z - float(slope[h]) * away
                err = max(err, abs(float(slope[h])) * float(away.max()) * 2.0 ** -22)
            z = z.masked_fill(~ok, -math.inf)
            lse[t:t + n, h] = torch.logsumexp(z, -1)
            w = torch.exp(z - lse[t:t + n, h, None])
            out[t:t + n, h], mag[t:t + n, h] = w @ v[:, h // group], w @ v[:, h // group].abs()
        t += n
    return out, lse, mag, 3 * err


CALLS = [("f32", 2, 64, 1, [5, 40], [100, 7]), ("f32", 1, 128, 2, [33], [400]), ("bf16", 2, 128, 1, [1, 3], [70, 300]), ("bf16", 2, 64, 3, [50], [111])]


def attend(c, q, group, cap, slope, scale):
    out, lse = torch.zeros(c.T, c.nh * group * c.hd, dtype=q.dtype, device=DEV), torch.zeros(c.T, c.nh * group, device=DEV)
    c.ctx.attend_ruled(0, c.lens, c.d_past, c.d_table, q, out, block=1, cap=cap, scale=scale, lse=lse,
                       slope=None if slope is None else torch.tensor(slope, device=DEV))
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("cap", [1e-3, 0.5, 2.0, 30.0, 1e3, 1e5, 1e6, 1e8, 1e30, 8e37])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("call", range(len(CALLS)))
def test_against_the_definition(cache_ops, call, bias, cap):
    dtype, nh, hd, G, lens, past = CALLS[call]
    c = cache_ops.Cache(dtype, nh, hd, lens, past, seed=call)
    slope, scale = [0.01 * (h + 1) for h in range(nh * G)] if bias else None, 1 / math.sqrt(hd)
    q = c.randn(c.T, nh * G * hd, scale=1.5)
    out, lse = attend(c, q, G, cap, slope, scale)
    ref, ref_lse, mag, err = definition(c, q, G, cap, slope, scale)
    e = 2 * err + 2.0 ** -19
    assert ((lse.cpu().double() - ref_lse).abs() <= e + 2.0 ** -21 * ref_lse.abs()).all()
    # (more than 32 rows: weights rounded to bfloat16)
    weight = 0.0 if dtype == "f32" else 2.0 ** -8 if max(lens) * G > 32 else 2.0 ** -15
    bar = cache_ops.HALF_STEP[dtype] * ref.abs() + (weight + e) * mag + 1e-30
    got = out.cpu().double().reshape(ref.shape)
    assert ((got - ref).abs() <= bar).all(), float(((got - ref).abs() / bar).max())
    c.close()


@pytest.mark.parametrize("call", range(len(CALLS)))
def test_scores_at_the_cap_and_far_below_it(cache_ops, call):
    """Scores of 1e9 and of infinity are the cap, both ways; a cap far above the scores leaves them, a scale far above the cap leaves signs."""
    dtype, nh, hd, G, lens, past = CALLS[call]
    c = cache_ops.Cache(dtype, nh, hd, lens, past, seed=call)
    q = c.randn(c.T, nh * G * hd, scale=1.5)
    plain, plain_lse = attend(c, q, G, 0.0, None, 0.0)
    for cap in (1e12, 8e37):
        out, lse = attend(c, q, G, cap, None, 0.0)
        # two roundings of scores of 30 at most, and what they change in sums and weights
        assert (lse - plain_lse).abs().max() <= 2.0 ** -17
        assert (out.double() - plain.double()).abs().max() <= (2.0 ** -7 if dtype == "bf16" else 2.0 ** -16) * 8
    sign, sign_lse = attend(c, q, G, 3.0, None, 1e9)      # +-3, but for the few products that are next to nothing
    again, again_lse = attend(c, q, G, 3.0, None, 1.6e38)
    for o, l in ((sign, sign_lse), (again, again_lse)):
        assert torch.isfinite(o).all() and torch.isfinite(l).all()
        n = torch.tensor([p + i + 1.0 for k, p in zip(lens, past) for i in range(k)], device=DEV)[:, None]
        assert (l <= 3.0 + n.log() + 2.0 ** -18).all() and (l >= -3.0 + n.log() - 2.0 ** -18).all()
    tiny, tiny_lse = attend(c, q, G, 1e-30, None, 1.6e38)      # weights alike
    assert (tiny_lse - n.log()).abs().max() <= 2.0 ** -19
    c.close()


@pytest.mark.parametrize("cap", [5.0, 30.0])
def test_a_capped_score_is_its_own(cache_ops, cap):
    """What lies in keys that nobody sees, and behind the last one, however large, changes no bit."""
    for dtype, nh, hd, G, lens, past in CALLS + [("bf16", 16, 128, 1, [2600], [300])]:
        c = cache_ops.Cache(dtype, nh, hd, lens, past, seed=11)
        q, total = c.randn(c.T, nh * G * hd, scale=1.5), lens[0] + past[0]
        out, lse = (torch.zeros(2, c.T, nh * G * w, dtype=t, device=DEV) for w, t in ((hd, q.dtype), (1, torch.float32)))
        first = torch.tensor([9] * c.T, dtype=torch.int32, device=DEV)
        for turn in range(2):
            c.ctx.attend_ruled(0, c.lens, c.d_past, c.d_table, q, out[turn], block=1, cap=cap, first=first, lse=lse[turn])
            torch.cuda.synchronize()
            c.set_rows(0, [0, 3, 8, total, total + 5], k=torch.full((5, nh, hd), 1e4))
        assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1])
        c.close()
