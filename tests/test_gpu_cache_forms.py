"""The paged cache's operators in their larger forms, and in settings of the rotation that change its angles."""
import math

import pytest

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
