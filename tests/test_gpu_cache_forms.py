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
