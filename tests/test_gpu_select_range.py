"""The choice of the best (row, token) pairs where logits are large, and where tokens are banned by a large negative number instead of -inf."""
import math

import pytest
import torch

from test_gpu_select import check, run

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def b():
    from paper_2510_08666_amd import binding
    return binding


def select(logits, score, keep):
    """[(score, row, token)] of every sequence, best first; the largest logit of a row is taken off before anything is added to what is left, so
    that 64 bits hold what the score and the sum of exponentials add to logits of any size."""
    out = []
    for s in range(logits.shape[0]):
        found = []
        for r in range(logits.shape[1]):
            base, z = float(score[s, r]), logits[s, r].double()
            m = float(z.max())
            if not math.isfinite(base) or m == -math.inf:
                continue
            x = (base - float(torch.exp(z - m).sum().log())) + (z - m)
            best = torch.sort(x, descending=True, stable=True)
            found += [(float(v), r, int(t)) for v, t in zip(best[0][:keep], best[1][:keep]) if v > -math.inf]
        found.sort(key=lambda f: (-f[0], f[1], f[2]))
        out.append(found[:keep])
    return out


def lowest(fill, dtype):
    return torch.finfo(dtype).min if fill == "lowest" else fill


@pytest.mark.parametrize("keep", [3, 24, 64])
@pytest.mark.parametrize("fill", ["lowest", -1e30, -1e20, -1e10, -1e9])
@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_banned_by_a_large_number(b, dtype, fill, keep):
    """Stretches of thousands of such logits beside ordinary ones, rows of little else, a row of nothing else."""
    g = torch.Generator().manual_seed(keep)
    z, fill = (3 * torch.randn(2, 6, 9000, generator=g)).to(dtype), lowest(fill, dtype)
    z[:, 1, 2048:6144] = fill
    z[:, 2] = fill
    z[0, 3, :] = fill
    z[0, 3, [5, 4100, 8999]] = torch.tensor([1.0, 0.5, 2.0], dtype=dtype)
    z[:, 4, 4000:] = fill
    z[:, :, 11::7] = fill
    score = -3 * torch.rand(2, 6, generator=g)
    score[1, 0], score[0, 5] = -math.inf, -math.inf
    check(run(b, z.to(DEV), score.to(DEV), keep), select(z, score, keep), keep)


@pytest.mark.parametrize("fill", ["lowest", -1e30, -1e10, -1e9, 1e30, 3e38])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_row_of_one_large_number(b, dtype, fill):
    """Every token of it shares the row's weight alike: the lowest tokens, at the score less the logarithm of the vocabulary."""
    z = torch.full((1, 1, 5000), lowest(fill, dtype), dtype=dtype)
    row, token, out = run(b, z.to(DEV), torch.tensor([[-2.0]], device=DEV), 9)
    assert (row == 0).all() and token[0].tolist() == list(range(9))
    assert (out.double() - (-2.0 - math.log(5000))).abs().max() <= 2.0 ** -20


@pytest.mark.parametrize("dtype", TYPES)
def test_banned_tokens_are_the_last_candidates(b, dtype):
    z = torch.full((1, 1, 4500), torch.finfo(dtype).min, dtype=dtype)
    z[0, 0, 4400], z[0, 0, 7] = 1.0, 0.0
    score = torch.tensor([[-1.0]])
    row, token, out = run(b, z.to(DEV), score.to(DEV), 6)
    assert (row == 0).all() and token[0].tolist() == [4400, 7, 0, 1, 2, 3]
    check((row, token, out), select(z, score, 6), 6)


@pytest.mark.parametrize("away", [40.0, -40.0, 1e3, -1e4, 1e6, 1e8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R", [4, 40])
def test_rows_of_different_sizes(b, dtype, away, R):
    """A constant added to a row changes nothing but what its logits lose when they are rounded."""
    g = torch.Generator().manual_seed(R)
    z = 3 * torch.randn(1, R, 6200, generator=g)
    z[0, 1] += away
    z[0, 3] += away / 2
    z, score = z.to(dtype), -torch.rand(1, R, generator=g)
    check(run(b, z.to(DEV), score.to(DEV), 32), select(z, score, 32), 32)
