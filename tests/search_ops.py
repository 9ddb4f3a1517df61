"""The operators of a search over several continuations, from their definitions on the CPU (64 bits), for their tests."""
import math

import torch

from cache_ops import HALF_STEP

PAGE = 16


def seen(rule, s, t, p, n_keys):
    """Which of n_keys positions the token t (of sequence s, at position p) sees, by the definition."""
    pre = rule["prefix"][s] if rule.get("prefix") is not None else 0
    j = torch.arange(n_keys)
    ok = torch.ones(n_keys, dtype=torch.bool)
    b, w = rule.get("block", 0), rule.get("window", 0)
    if b:
        ok &= j < (pre if p < pre else pre + ((p - pre) // b + 1) * b)
    if w:
        ok &= (j - p).abs() < w
    ok |= j < pre
    if rule.get("first") is not None:
        ok &= j >= rule["first"][t]
    if rule.get("end") is not None:
        ok &= j < rule["end"][t]
    return ok


def attention(c, q, group, rule, scale=None, layer=0):
    """out, lse, sum of p |v| per output, and a bound on a score's float32 error: of its product (hd + 4 roundings of its size), of the cap
    (the exponential and the reciprocal: a few 2^-24 of it) and of the bias (three roundings of it)."""
    pool = c.pool.cpu()
    nq = c.nh * group
    scale = scale or 1 / math.sqrt(c.hd)
    q = q.cpu().double().reshape(c.T, nq, c.hd)
    out, lse = torch.zeros(c.T, nq, c.hd, dtype=torch.float64), torch.full((c.T, nq), -math.inf, dtype=torch.float64)
    mag, err, t = torch.zeros_like(out), 0.0, 0
    cap, slope = rule.get("cap", 0.0), rule.get("slope")
    for s in range(c.ns):
        n, p = c.lens[s], c.past[s]
        k, v = c.rows(s, n + p, pool, layer)
        ok = torch.stack([seen(rule, s, t + i, p + i, n + p) for i in range(n)]) if n else torch.zeros(0, p, dtype=torch.bool)
        away = (torch.arange(n + p)[None] - torch.arange(p, p + n)[:, None]).abs().double()
        for h in range(nq):
            kh, vh = k[:, h // group], v[:, h // group]
            z = q[t:t + n, h] @ kh.t() * scale
            size = (q[t:t + n, h].abs() @ kh.abs().t() * scale)[ok].nan_to_num(0, 0, 0)
            e = float(size.max()) * (c.hd + 4) * 2.0 ** -24 if size.numel() else 0.0
            if cap:
                z = cap * torch.tanh(z / cap)
                e += cap * 2.0 ** -21
            if slope is not None:
                z = z - float(slope[h]) * away
                e += abs(float(slope[h])) * (float(away[ok].max()) if ok.any() else 0.0) * 2.0 ** -22
            err = max(err, e)
            z = z.masked_fill(~ok, -math.inf)
            some = ok.any(1)
            lse[t:t + n, h] = torch.where(some, torch.logsumexp(z, -1), -math.inf)
            w = torch.where(ok, torch.exp(z - torch.where(some, lse[t:t + n, h], 0.0)[:, None]), 0.0)
            if torch.isfinite(vh).all():
                out[t:t + n, h], mag[t:t + n, h] = w @ vh, w @ vh.abs()
            else:
                for i in range(n):      # row by row: only what the row sees takes part
                    out[t + i, h], mag[t + i, h] = w[i, ok[i]] @ vh[ok[i]], w[i, ok[i]] @ vh[ok[i]].abs()
        t += n
    return out, lse, mag, err


def check_attention(c, q, group, rule, out, lse=None, scale=None):
    """|error| <= half a step of the output + half a bfloat16 step of every weight (in front of the product with the values; none in
    float32) + twice the score's error and 2^-19 (exponentials and sums) of what the values weigh."""
    ref, ref_lse, mag, err = attention(c, q, group, rule, scale)
    e = 2 * err + 2.0 ** -19
    got = out.cpu().double()[:c.T].reshape(ref.shape)
    bar = HALF_STEP[c.dtype] * ref.abs() + (2.0 ** -8 if c.dtype == "bf16" else 0.0) * mag + e * mag + 1e-30
    bad = ~((got - ref).abs() <= bar) & ~(torch.isnan(got) & torch.isnan(ref)) & ~(got == ref)
    assert not bad.any(), (bad.nonzero()[:5], got[bad][:5], ref[bad][:5])
    if lse is not None:
        g = lse.cpu().double()[:c.T].reshape(ref_lse.shape)
        ok = ((g - ref_lse).abs() <= e + 2.0 ** -21 * ref_lse.abs()) | (g == ref_lse) | torch.isnan(ref_lse)
        assert ok.all(), (ref_lse[~ok][:5], g[~ok][:5])


def select(logits, score, keep, hold=None):
    """[(score, row, token)] of every sequence, best first."""
    out = []
    for s in range(logits.shape[0]):
        found = []
        for r in range(logits.shape[1]):
            base = float(score[s, r])
            if not math.isfinite(base):
                continue
            if hold is not None and int(hold[s, r]) >= 0:
                found.append((base, r, int(hold[s, r])))
                continue
            z = logits[s, r].double()
            z = torch.where(torch.isnan(z), -math.inf, z)
            m = float(z.max())
            if m == -math.inf:
                continue
            if m == math.inf:
                x = torch.where(z == math.inf, base - math.log(int((z == math.inf).sum())), -math.inf)
            else:
                x = base + (z - (m + torch.exp(z - m).sum().log()))
            best = torch.sort(x, descending=True, stable=True)
            found += [(float(v), r, int(t)) for v, t in zip(best[0][:keep], best[1][:keep]) if v > -math.inf]
        found.sort(key=lambda f: (-f[0], f[1], f[2]))
        out.append(found[:keep])
    return out


def fork(table, held, length, refs, parent, room, rewrite, columns, limit):
    """One sequence after the other: tables, lengths, held columns, counts, [(from, to)] pages to copy, free pages that are missing."""
    n_pages = len(refs)
    new_refs = list(refs)
    for s in range(len(held)):
        for c in range(held[s]):
            new_refs[table[s][c]] -= 1
    free = [p for p in range(n_pages) if refs[p] <= 0]
    seen_parents, rows, lens, helds, copies, missing = set(), [], [], [], [], 0
    for p in parent:
        p = p if 0 <= p < len(held) else -1
        n = min(max(length[p], 0), limit) if p >= 0 else 0
        need = min(-(-(n + room) // PAGE), columns)
        own, row = max(0, n - rewrite) // PAGE, []
        for c in range(need):
            page = table[p][c] if p >= 0 and c < held[p] else -1
            if c < own:
                row.append(page)
            elif page >= 0 and p not in seen_parents and refs[page] == 1:
                row.append(page)
            elif not free:
                missing += 1
                row.append(-1)
            else:
                row.append(free.pop(0))
                if page >= 0 and c * PAGE < n:
                    copies.append((page, row[-1]))
        seen_parents.add(p)
        for page in row:
            if page >= 0:
                new_refs[page] += 1
        rows.append(row + [-1] * (columns - len(row)))
        lens.append(n)
        helds.append(need)
    return rows, lens, helds, new_refs, copies, missing


def compact(refs):
    """Every page's new number (-1: free), and the pages that move."""
    used = [p for p, r in enumerate(refs) if r > 0]
    front = len(used)
    free = [p for p in range(front) if refs[p] <= 0]
    moved = [-1] * len(refs)
    movers = [p for p in used if p >= front]
    for p in used:
        moved[p] = p
    for p, to in zip(movers, free):
        moved[p] = to
    return moved, movers
