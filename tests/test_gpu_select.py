"""The choice of the best (row, token) pairs against its definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32


@pytest.fixture(scope="module")
def m():
    import search_ops
    from paper_2510_08666_amd import binding
    return binding, search_ops


def run(b, logits, score, keep, hold=None):
    ns, R, V = logits.shape
    row, token = (torch.full((ns, keep), -7, dtype=I32, device=DEV) for _ in range(2))
    out, scratch = torch.full((ns, keep), 7.0, device=DEV), b.beam_scratch(ns, R, V, keep)
    scratch.fill_(255)
    b.beam_select(logits, score, row, token, out, scratch, hold=hold)
    torch.cuda.synchronize()
    return row.cpu(), token.cpu(), out.cpu()


def check(got, ref, keep):
    """Scores within half a step of float32 of the 64-bit ones and what the slices' sums of exponentials (float32, 2^-20 of them at most:
    exponentials, and 32 + 6 + 4 additions that lose half a step each) leave in the logarithm; pairs equal wherever neighbours are further apart."""
    row, token, score = got
    for s, want in enumerate(ref):
        n = len(want)
        assert (row[s, n:] == -1).all() and (token[s, n:] == -1).all() and (score[s, n:] == -math.inf).all(), s
        values = [w[0] for w in want]
        for k in range(n):
            bar = 2.0 ** -24 * abs(values[k]) + 2.0 ** -20
            assert score[s, k] == values[k] or abs(float(score[s, k]) - values[k]) <= bar, (s, k, float(score[s, k]), values[k])
            near = [w for w in want if w[0] == values[k] or abs(w[0] - values[k]) <= 2 * bar]
            if all(w[0] == values[k] and w[1] == want[k][1] for w in near):      # (equal in one row: the order is exact)
                if k < n - 1 or n < keep or len(near) > 1:
                    assert (int(row[s, k]), int(token[s, k])) == want[k][1:], (s, k, want[k], int(row[s, k]), int(token[s, k]))


@pytest.mark.parametrize("keep", [1, 5, 16, 64])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ns,R,V", [(1, 1, 1), (2, 3, 63), (1, 4, 8192), (3, 7, 8193), (1, 2, 50001), (2, 33, 4096), (1, 300, 257)])
def test_against_the_definition(m, ns, R, V, dtype, keep):
    b, ops = m
    g = torch.Generator().manual_seed(V + R + keep)
    z = (3 * torch.randn(ns, R, V, generator=g)).to(dtype)
    z[..., ::7] = -math.inf
    score = -5 * torch.rand(ns, R, generator=g)
    score[:, 2::4] = -math.inf
    hold = torch.full((ns, R), -1, dtype=I32)
    hold[:, 1::5] = 2
    ref = ops.select(z, score, keep, hold)
    check(run(b, z.to(DEV), score.to(DEV), keep, hold.to(DEV)), ref, keep)


def test_a_whole_vocabulary(m):
    b, ops = m
    g = torch.Generator().manual_seed(3)
    z = (2.5 * torch.randn(2, 6, 157184, generator=g)).bfloat16()
    score = -5 * torch.rand(2, 6, generator=g)
    check(run(b, z.to(DEV), score.to(DEV), 32), ops.select(z, score, 32), 32)


@pytest.mark.parametrize("V,R,keep", [(20000, 3, 64), (9000, 1, 7), (300, 1000, 64), (1, 1024, 64)])
def test_all_equal(m, V, R, keep):
    """Thousands of equal candidates, more than any list holds: the lowest rows and tokens."""
    b, ops = m
    z, score = torch.full((1, R, V), 1.5, dtype=torch.bfloat16), torch.full((1, R), -2.0)
    row, token, out = run(b, z.to(DEV), score.to(DEV), keep)
    want = [(i // V, i % V) for i in range(keep)]
    assert list(zip(row[0].tolist(), token[0].tolist())) == want
    assert (out - (-2.0 - math.log(V))).abs().max() <= 2.0 ** -20


def test_ties_of_a_coarse_grid_and_of_equal_rows(m):
    """Logits on a grid of quarters, the same row several times: equal scores are common, the lower row and token come first."""
    b, ops = m
    g = torch.Generator().manual_seed(11)
    z = (4 * torch.randn(1, 1, 9001, generator=g)).mul(4).round().div(4).clamp(max=8.0)
    z = z.expand(2, 5, 9001).contiguous()
    score = torch.tensor([[-1.0] * 5, [-1.0, -math.inf, -1.0, -1.0, -2.0]])
    row, token, out = run(b, z.to(DEV), score.to(DEV), 40)
    for s, w in enumerate(ops.select(z, score, 40)):
        assert list(zip(row[s].tolist(), token[s].tolist())) == [x[1:] for x in w]


def test_odd_values(m):
    """NaN and -inf are no candidates, +inf share the row's weight, rows of nothing and dead rows leave nothing (and are not read)."""
    b, ops = m
    g = torch.Generator().manual_seed(4)
    z = torch.randn(1, 8, 5000, generator=g)
    z[0, 0, 17], z[0, 0, 4999] = math.inf, math.inf
    z[0, 1] = -math.inf
    z[0, 2, 3:] = math.nan
    z[0, 3] = math.nan
    z[0, 5, 5:] = -math.inf
    z[0, 7, 100] = -math.inf
    score = torch.tensor([[-30.0, 0.0, -1.0, 0.0, math.nan, -2.0, -math.inf, -3.0]])
    ref = ops.select(z, score, 24)
    check(run(b, z.to(DEV), score.to(DEV), 24), ref, 24)
    dead = torch.full((1, 8), -math.inf, device=DEV)
    dead[0, 1:4] = torch.tensor([math.inf, math.nan, math.inf])
    row, token, out = run(b, z.to(DEV), dead, 3)
    assert (row == -1).all() and (token == -1).all() and (out == -math.inf).all()
    hold = torch.full((1, 8), 4, dtype=I32, device=DEV)
    score = torch.tensor([[-1.0, -3.0, -1.0, -math.inf, -0.5, -4.0, -9.0, -2.0]], device=DEV)
    row, token, out = run(b, z.to(DEV), score, 9, hold)
    assert row[0].tolist() == [4, 0, 2, 7, 1, 5, 6, -1, -1] and token[0].tolist() == [4] * 7 + [-1, -1]
    assert out[0, :7].tolist() == [-0.5, -1.0, -1.0, -2.0, -3.0, -4.0, -9.0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("skew,stride", [(0, 1000), (1, 1001), (5, 1003), (3, 1008)])
def test_strides_and_alignment(m, dtype, skew, stride):
    b, ops = m
    g = torch.Generator().manual_seed(stride)
    flat = torch.randn(skew + 6 * stride + 9, generator=g).to(dtype)
    flat[:skew] = 50.0
    rows = flat[skew:skew + 6 * stride].view(2, 3, stride)
    rows[..., 997:] = 60.0      # behind the rows: never a candidate
    flat[skew + 6 * stride:] = 70.0
    score = -torch.rand(2, 3, generator=g)
    check(run(b, flat.to(DEV)[skew:skew + 6 * stride].view(2, 3, stride)[..., :997], score.to(DEV), 11), ops.select(rows[..., :997], score, 11), 11)


def test_streams_and_graphs(m):
    b, ops = m
    g = torch.Generator().manual_seed(6)
    ns, R, V, keep = 2, 5, 30000, 8
    z, score = torch.zeros(ns, R, V, device=DEV), torch.zeros(ns, R, device=DEV)
    row, token, out = torch.zeros(ns, keep, dtype=I32, device=DEV), torch.zeros(ns, keep, dtype=I32, device=DEV), torch.zeros(ns, keep, device=DEV)
    scratch, s = b.beam_scratch(ns, R, V, keep), torch.cuda.Stream()
    with torch.cuda.stream(s):
        b.beam_select(z, score, row, token, out, scratch)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            b.beam_select(z, score, row, token, out, scratch)
    for turn in range(4):
        hz, hs = 3 * torch.randn(ns, R, V, generator=g), -torch.rand(ns, R, generator=g)
        z.copy_(hz)
        score.copy_(hs)
        eager = run(b, z, score, keep)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(row.cpu(), eager[0]) and torch.equal(token.cpu(), eager[1]) and torch.equal(out.cpu(), eager[2])
        check(eager, ops.select(hz, hs, keep), keep)


def test_refusals(m):
    b, _ = m
    z, score = torch.zeros(1, 2, 9, device=DEV), torch.zeros(1, 2, device=DEV)
    row, token, out, scratch = torch.zeros(1, 3, dtype=I32, device=DEV), torch.zeros(1, 3, dtype=I32, device=DEV), torch.zeros(1, 3, device=DEV), b.beam_scratch(1, 2, 9, 3)
    b.beam_select(z, score, row, token, out, scratch)
    for bad in (dict(logits=z[0]), dict(logits=z.half()), dict(score=score[:, :1]), dict(row=row.long()), dict(token=token[:, :2]), dict(score_out=out.cpu()),
                dict(scratch=scratch.int()), dict(hold=score), dict(logits=torch.zeros(1, 9, 2, device=DEV).transpose(1, 2)), dict(logits=None), dict(row=None)):
        with pytest.raises(ValueError):
            b.beam_select(**{**dict(logits=z, score=score, row=row, token=token, score_out=out, scratch=scratch), **bad})
    with pytest.raises(b.DinferError):
        b.beam_select(z, score, row, token, out, scratch[:scratch.numel() - 1])
    with pytest.raises(b.DinferError):
        b.beam_select(z, score, row, row, out, scratch)
    torch.cuda.synchronize()


@pytest.mark.parametrize("ns,R,V,live,keep", [(4, 1, 4096, 1, 32), (2, 64, 9000, 3, 64), (1, 512, 1500, 512, 32), (3, 1, 100, 1, 64), (2, 40, 10, 40, 64), (1, 130, 2100, 70, 64)])
def test_few_chunks_with_candidates(m, ns, R, V, live, keep):
    """Fewer than n_keep stretches of logits that hold a candidate, many of them in each; many short rows."""
    b, ops = m
    g = torch.Generator().manual_seed(V)
    z, score = 3 * torch.randn(ns, R, V, generator=g), -torch.rand(ns, R, generator=g)
    for s in range(ns):
        score[s, torch.randperm(R, generator=g)[live:]] = -math.inf
    check(run(b, z.to(DEV), score.to(DEV), keep), ops.select(z, score, keep), keep)
