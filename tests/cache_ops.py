"""A context with a random page pool, and the paged cache's operators in float64 on the CPU, for their tests."""
import math

import numpy as np
import torch

import dinfer_inputs as di
from paper_2510_08666_amd import binding

PAGE = 16
DEV = "cuda:0"
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}      # finfo.eps / 2
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


class Cache:
    def __init__(self, dtype, heads, head_dim, lens, past, layers=1, seed=0, spare=2, max_pos=None, room=0, columns=0):
        self.dtype, self.nh, self.hd, self.L = dtype, heads, head_dim, layers
        self.lens, self.past, self.ns, self.T = list(lens), list(past), len(lens), sum(lens)
        g = torch.Generator().manual_seed(seed)
        self.g = g
        need = [-(-(l + p + room) // PAGE) + 1 for l, p in zip(lens, past)]
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((self.ns, max(need + [columns])), -1, dtype=torch.int32)      # entries that no call may follow
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.free = order[at:]
        cfg = di.configs.scaled(di.model_preset("tiny"), n_layers=layers, hidden=64, n_heads=heads, head_dim=head_dim, n_experts=1, top_k=1,
                                moe_inter=64, vocab=64, dtype=dtype)
        self.cfg, self.max_pos = cfg, max_pos or max(need + [columns]) * PAGE
        self.ctx = binding.Context(cfg, self.n_pages, self.ns, 64, self.max_pos)
        self.pool = self.ctx.kv.view(TYPE[dtype]).view(layers, self.n_pages, 2, -1)
        self.pool.copy_(torch.randn(self.pool.shape, generator=g).to(TYPE[dtype]))
        self.d_table, self.d_past = self.table.to(DEV), torch.tensor(past, dtype=torch.int32, device=DEV)

    def randn(self, *shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=self.g)).to(TYPE[self.dtype]).to(DEV)

    def close(self):
        self.ctx.close()

    # ---- the pool as rows, float64 [position][head][feature]
    def views(self, pool, layer=0):
        kb = 32 // pool.element_size()
        return (pool[layer, :, 0].view(self.n_pages, self.nh, self.hd // kb, PAGE, kb),
                pool[layer, :, 1].view(self.n_pages, self.nh, self.hd, PAGE))

    def rows(self, s, n, pool=None, layer=0, table=None):
        pool = self.pool.cpu() if pool is None else pool
        K, V = self.views(pool, layer)
        table = self.table if table is None else table
        pg = table[s, :-(-n // PAGE)].long() if n else torch.zeros(0, dtype=torch.long)
        k = K[pg].permute(0, 3, 1, 2, 4).reshape(-1, self.nh, self.hd)[:n].double()
        v = V[pg].permute(0, 3, 1, 2).reshape(-1, self.nh, self.hd)[:n].double()
        return k, v

    def set_rows(self, s, positions, k=None, v=None, layer=0):
        """Overwrites cached rows (device pool) with [n][head][feature] values."""
        K, V = self.views(self.pool, layer)
        for i, p in enumerate(positions):
            pg = int(self.table[s, p // PAGE])
            if k is not None:
                K[pg, :, :, p % PAGE] = k[i].to(self.pool.dtype).to(DEV).view(self.nh, K.shape[2], K.shape[4])
            if v is not None:
                V[pg, :, :, p % PAGE] = v[i].to(self.pool.dtype).to(DEV)

    # ---- references
    def attention(self, q, group, words=None, scale=None, layer=0):
        """out, lse, weights per sequence [token][query head][key], sum p |v|, and a bound on a score's float32 error."""
        pool = self.pool.cpu()
        nq = self.nh * group
        scale = scale or 1 / math.sqrt(self.hd)
        q = q.cpu().double().reshape(self.T, nq, self.hd)
        out, lse = torch.zeros(self.T, nq, self.hd, dtype=torch.float64), torch.full((self.T, nq), -math.inf, dtype=torch.float64)
        mag, err, weights, t = torch.zeros_like(out), 0.0, [], 0
        for s in range(self.ns):
            n, p = self.lens[s], self.past[s]
            k, v = self.rows(s, n + p, pool, layer)
            hidden = torch.zeros(n, n + p, dtype=torch.bool)
            if words is not None:
                for i in range(n):
                    hidden[i, p:] = torch.tensor([not (words[t + i] >> j) & 1 for j in range(n)], dtype=torch.bool)
            w = torch.zeros(n, nq, n + p, dtype=torch.float64)
            for h in range(nq):
                z = (q[t:t + n, h] @ k[:, h // group].t() * scale).masked_fill(hidden, -math.inf)
                size = (q[t:t + n, h].abs() @ k[:, h // group].abs().t() * scale)[~hidden]
                if size.numel():
                    err = max(err, float(size.nan_to_num(0, 0, 0).max()) * (self.hd + 4) * 2.0 ** -24)
                lse[t:t + n, h] = torch.logsumexp(z, -1) if n + p else -math.inf
                w[:, h] = torch.where(hidden, 0.0, torch.exp(z - lse[t:t + n, h, None]))
                vv = v[:, h // group]
                for i in range(n):           # row by row: only what the row sees takes part
                    see = ~hidden[i]
                    out[t + i, h] = w[i, h, see] @ vv[see]
                    mag[t + i, h] = w[i, h, see] @ vv[see].abs()
            weights.append(w)
            t += n
        return out, lse, weights, mag, err


def tree_words(g, lens):
    words = []
    for l in lens:
        seen = []
        for i in range(l):
            parent = i - 1 - int(torch.randint(0, 4, (1,), generator=g))
            seen.append((1 << i) | (seen[parent] if parent >= 0 else 0))
        words += seen
    return words


def word_tensor(words):
    return torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device=DEV)


def check_attention(c, q, group, out, lse, words=None, scale=None):
    """|error| <= half a step of the output + half a bfloat16 step of every weight (their rounding in front of the second
    product; none in float32) + the float32 error of scores, exponentials (relative 2^-21) and sums."""
    ref, ref_lse, _, mag, err = c.attention(q, group, words, scale)
    e = 2 * err + 2.0 ** -19
    got = out.cpu().double().reshape(ref.shape)
    bar = HALF_STEP[c.dtype] * ref.abs() + (2.0 ** -8 if c.dtype == "bf16" else 0.0) * mag + e * mag + 1e-30
    bad = ~((got - ref).abs() <= bar) & ~(torch.isnan(got) & torch.isnan(ref)) & ~((got == ref))
    assert not bad.any(), (bad.nonzero()[:5], got[bad][:5], ref[bad][:5])
    if lse is not None:
        d = (lse.cpu().double().reshape(ref_lse.shape) - ref_lse).abs()
        ok = (d <= e + 2.0 ** -21 * ref_lse.abs()) | (lse.cpu().reshape(ref_lse.shape) == ref_lse) | torch.isnan(ref_lse)
        assert ok.all(), (ref_lse[~ok][:5], lse.cpu()[~ok][:5])
