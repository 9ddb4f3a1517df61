"""Attention over the paged cache, value for value: outputs within their own rounding of float64, and cached values that are no finite
numbers, which every row sees, wherever in the key range they lie."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import cache_ops
    return cache_ops


def check(c, q, group, out, lse, words=None):
    """|error| <= half a step of the output + 2^-15 of every weight (in bfloat16 weights enter the second product as two planes: what is
    left of the second one's rounding is 2^-7 * 2^-8) + the float32 error of scores, exponentials (relative 2^-21) and sums.  NaN and
    infinities are where the definition has them, in the outputs and in the normalisers."""
    import cache_ops
    import torch
    ref, ref_lse, _, mag, err = c.attention(q, group, words)
    e = 2 * err + 2.0 ** -19 + (2.0 ** -15 if c.dtype == "bf16" else 0.0)
    got, norm = out.cpu().double().reshape(ref.shape), lse.cpu().double().reshape(ref_lse.shape)

    def ok(x, r, bar):
        return (torch.isfinite(r) & ((x - r).abs() <= bar)) | (x == r) | (torch.isnan(x) & torch.isnan(r))

    bad = ~ok(got, ref, cache_ops.HALF_STEP[c.dtype] * ref.abs() + e * mag + 1e-30)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:5], got[bad][:5], ref[bad][:5])
    bad = ~ok(norm, ref_lse, 2 * err + 2.0 ** -19 + 2.0 ** -21 * ref_lse.abs())
    assert not bad.any(), (bad.nonzero()[:5], norm[bad][:5], ref_lse[bad][:5])
    return ref, ref_lse


# Forms: 30 rows per cache head (one row tile), 60 and 90 (two), and, with many cache heads and page-table rows of 32768 positions, 90 and 270
# rows in the form of many rows with four and eight waves.  900 cached positions are cut into parts, 300 are not.
FORMS = [("bf16", 4, 1, 0), ("bf16", 4, 2, 0), ("bf16", 4, 3, 0), ("bf16", 36, 3, 2048), ("bf16", 20, 9, 2048), ("f32", 4, 1, 0), ("f32", 4, 3, 0)]


def case(m, form, hd, past, seed):
    import torch
    dtype, heads, group, columns = form
    c = m.Cache(dtype, heads, hd, [30, 9], [past, 3], seed=seed, columns=columns)
    q = c.randn(c.T, heads * group * hd, scale=1.5)
    return c, q, torch.empty_like(q), torch.empty(c.T, heads * group, device=m.DEV)


def words_of(m, c, kind):
    return {"none": lambda: None, "tree": lambda: m.tree_words(c.g, c.lens), "causal": lambda: [(2 << j) - 1 for l in c.lens for j in range(l)]}[kind]()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("past", [5, 300, 900])
@pytest.mark.parametrize("kind", ["none", "tree"])
def test_outputs_are_rounded_once(m, form, hd, past, kind):
    c, q, out, lse = case(m, form, hd, past, 60 + past)
    words = words_of(m, c, kind)
    c.ctx.attend(0, c.lens, c.d_past, c.d_table, q, out, visible=None if words is None else m.word_tensor(words), lse=lse)
    check(c, q, form[2], out, lse, words)
    c.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("past", [0, 37, 900])
def test_hidden_values_in_the_form_of_many_rows(m, hd, past):
    """What a token does not see does not reach it in the form of many rows with four waves either."""
    import test_gpu_cache_ops
    test_gpu_cache_ops.hidden_case(m, "bf16", 36, hd, past, 3, columns=2048)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("past", [70, 300, 900])
@pytest.mark.parametrize("kind", ["none", "tree"])
def test_cached_values_that_are_not_finite(m, form, hd, past, kind):
    """NaN and both infinities in cached values, one position in every run of 32 (so in every turn and at every part's start) and the last one
    cached, each in features of its own: they reach those features of every row and no other."""
    import torch
    c, q, out, lse = case(m, form, hd, past, 70 + past)
    at = sorted({min(32 * i + 5 * i % 32, past - 1) for i in range(-(-past // 32))} | {past - 1, past // 64 * 64})
    odd = [math.nan, math.inf, -math.inf]
    planted = {}
    for i, p in enumerate(at):
        _, v = c.rows(0, past)
        row = v[p].clone()
        row[:, 2 * i] = odd[i % 3]
        if i % 2:
            row[:, 2 * i + 1] = odd[(i + 1) % 3]
        planted[p] = row
    c.set_rows(0, list(planted), v=torch.stack(list(planted.values())))
    words = words_of(m, c, kind)
    c.ctx.attend(0, c.lens, c.d_past, c.d_table, q, out, visible=None if words is None else m.word_tensor(words), lse=lse)
    ref, ref_lse = check(c, q, form[2], out, lse, words)
    assert torch.isnan(ref[:30]).any() and torch.isinf(ref[:30]).any() and torch.isfinite(ref[:30]).any() and torch.isfinite(ref[30:]).all()
    assert torch.isfinite(ref_lse).all()
    c.close()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("at,kind", [(5, "tree"), (479, "none"), (703, "tree"), (899, "none")])
def test_cached_keys_that_are_not_numbers(m, form, hd, at, kind):
    """A NaN in one cache head's key at a cached position makes that head's rows of that sequence NaN, and their normalisers; every other
    row is as it should be."""
    import torch
    dtype, heads, group, _ = form
    c, q, out, lse = case(m, form, hd, 900, 80 + at)
    k, _ = c.rows(0, 900)
    row = k[at].clone()
    row[1, 7] = math.nan
    c.set_rows(0, [at], k=row[None])
    words = words_of(m, c, kind)
    c.ctx.attend(0, c.lens, c.d_past, c.d_table, q, out, visible=None if words is None else m.word_tensor(words), lse=lse)
    check(c, q, group, out, lse, words)
    hit = torch.zeros(c.T, heads * group, dtype=torch.bool)
    hit[:30, group:2 * group] = True
    assert torch.equal(torch.isnan(lse).cpu(), hit) and torch.equal(torch.isnan(out).view(c.T, heads * group, hd).all(-1).cpu(), hit)
    c.close()
