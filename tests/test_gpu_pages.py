"""Sequences that fork, and pools that are packed, against a bookkeeping that does one thing after the other."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32
PAGE = 16


@pytest.fixture(scope="module")
def m():
    import dinfer_inputs as di
    import search_ops
    from paper_2510_08666_amd import binding
    return di, binding, search_ops


def ints(x):
    return torch.tensor(x, dtype=I32, device=DEV)


class Pool:
    def __init__(self, m, n_pages, dtype="bf16", heads=2, head_dim=64, layers=2, seed=0, max_pos=2048, max_seqs=64):
        di, b, _ = m
        cfg = di.configs.scaled(di.model_preset("tiny"), n_layers=layers, hidden=64, n_heads=heads, head_dim=head_dim, n_experts=1, top_k=1,
                                moe_inter=64, vocab=64, dtype=dtype)
        self.ctx = b.Context(cfg, n_pages, max_seqs, 64, max_pos)
        self.n, self.max_pos = n_pages, max_pos
        self.kv = self.ctx.kv.view(I32).view(layers, n_pages, -1)
        self.kv.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, self.kv.shape, generator=torch.Generator().manual_seed(seed)))

    def fork(self, parent, length, held, table, refs, room, rewrite, columns, states=()):
        n = len(parent)
        out = dict(d_new_len=torch.full((n,), -9, dtype=I32, device=DEV), d_new_held=torch.full((n,), -9, dtype=I32, device=DEV),
                   d_new_page_table=torch.full((n, columns), -9, dtype=I32, device=DEV), new_refs=torch.full((self.n,), -9, dtype=I32, device=DEV),
                   short=torch.full((1,), -9, dtype=I32, device=DEV))
        old = (ints(length), ints(held), ints(table)) if len(held) else (None, None, None)
        self.ctx.kv_fork(ints(parent), *old, ints(refs), room=room, rewrite=rewrite, states=states, **out)
        torch.cuda.synchronize()
        return {k: v.cpu().tolist() for k, v in out.items()}

    def close(self):
        self.ctx.close()


def draw(rng, n_pages, n_old, longest, old_columns):
    """Old sequences, some of whose pages are held by others too."""
    table, held, length, refs = [], [], [], [0] * n_pages
    free = list(range(n_pages))
    rng.shuffle(free)
    for s in range(n_old):
        n = rng.choice([0, 1, 15, 16, 17, rng.randint(0, longest)])
        h = min(-(-n // PAGE) + rng.randint(0, 2), old_columns)
        row = []
        if s and rng.random() < 0.6:      # begins like an older one
            t = rng.randrange(s)
            row = table[t][:rng.randint(0, min(held[t], h))]
        while len(row) < h:
            row.append(free.pop())
        for p in row:
            refs[p] += 1
        table.append(row + [rng.choice([-1, 10 ** 6]) for _ in range(old_columns - h)])
        held.append(h)
        length.append(min(n, h * PAGE))
    return table, held, length, refs


@pytest.mark.parametrize("dtype,heads,head_dim,layers", [("bf16", 2, 64, 2), ("f32", 3, 64, 1), ("bf16", 5, 128, 3)])
def test_fork_against_one_after_the_other(m, dtype, heads, head_dim, layers):
    _, b, ops = m
    rng = random.Random(heads)
    pool = Pool(m, 300, dtype, heads, head_dim, layers)
    for turn in range(30):
        n_old, n_new = rng.choice([1, 2, 7, 20]), rng.choice([1, 2, 8, 24])
        old_columns, columns = rng.randint(9, 20), rng.randint(9, 20)
        table, held, length, refs = draw(rng, 300, n_old, 140, old_columns)
        parent = [rng.choice([-1, 99, rng.randrange(n_old), rng.randrange(n_old)]) for _ in range(n_new)]
        room, rewrite = rng.choice([0, 1, 16, 33]), rng.choice([0, 0, 1, 16, 40])
        limit = min(pool.max_pos, 16 * min(old_columns, columns))
        rows, lens, helds, new_refs, copies, missing = ops.fork(table, held, length, refs, parent, room, rewrite, columns, limit)
        before = pool.kv.cpu()
        words, marks = torch.randint(0, 99, (n_old, 37), dtype=I32, device=DEV), torch.rand(n_old, 4100, device=DEV)
        new_words, new_marks = torch.full((n_new, 37), -5, dtype=I32, device=DEV), torch.full((n_new, 4100), -5.0, device=DEV)
        got = pool.fork(parent, length, held, table, refs, room, rewrite, columns, [(words, new_words), (marks, new_marks)])
        assert got["short"] == [missing], turn
        if missing:
            assert all(set(got[k]) == {-9} for k in ("d_new_len", "d_new_held", "new_refs")) and torch.equal(pool.kv.cpu(), before)
            assert (new_words == -5).all() and set(sum(got["d_new_page_table"], [])) == {-9}
            continue
        assert got["d_new_len"] == lens and got["d_new_held"] == helds and got["new_refs"] == new_refs, turn
        assert got["d_new_page_table"] == rows, turn
        for a, z in copies:
            before[:, z] = before[:, a]
        assert torch.equal(pool.kv.cpu(), before), turn
        for i, p in enumerate(parent):
            alive = 0 <= p < n_old
            assert torch.equal(new_words[i], words[p]) if alive else (new_words[i] == 0).all()
            assert torch.equal(new_marks[i], marks[p]) if alive else (new_marks[i] == 0).all()
    pool.close()


def test_fork_short_of_pages_and_out_of_nothing(m):
    _, b, ops = m
    pool = Pool(m, 20, max_seqs=8)
    got = pool.fork([-1, -1, 5], [], [], [], [0, 1, 0, 0] + [1] * 12 + [0] * 4, 20, 0, 3)
    assert got["short"] == [0] and got["d_new_page_table"] == [[0, 2, -1], [3, 16, -1], [17, 18, -1]] and got["d_new_len"] == [0] * 3
    before = pool.kv.cpu()
    new = torch.full((3, 2), 4.0, device=DEV)
    got = pool.fork([0, 0, 0], [17], [2], [[0, 1]], [1, 1] + [3] * 16 + [0, 0], 16, 0, 9, [(torch.zeros(1, 2, device=DEV), new)])
    # 17 positions and 16 more: 3 columns, the first one shared; the first child keeps column 1
    assert got["short"] == [3] and (new == 4).all() and set(got["new_refs"]) == {-9} and torch.equal(pool.kv.cpu(), before)
    got = pool.fork([0, -1, 0], [17], [2], [[0, 1]], [1, 1] + [3] * 14 + [0] * 4, 0, 0, 9)
    assert got["short"] == [0] and got["d_new_page_table"] == [[0, 1] + [-1] * 7, [-1] * 9, [0, 16] + [-1] * 7] and got["d_new_held"] == [2, 0, 2]
    assert got["new_refs"] == [2, 1] + [3] * 14 + [1, 0, 0, 0] and torch.equal(pool.kv[:, 16].cpu(), before[:, 1])
    pool.close()


@pytest.mark.parametrize("n_pages", [1, 63, 64, 65, 1000])
def test_compact_against_one_after_the_other(m, n_pages):
    _, b, ops = m
    rng = random.Random(n_pages)
    pool = Pool(m, n_pages, layers=2, heads=1)
    for turn in range(8):
        share = rng.choice([0.0, 0.1, 0.5, 0.9, 1.0])
        used = [p for p in range(n_pages) if rng.random() < share]
        refs = [0] * n_pages
        columns, rows, held = max(len(used), 1) + 1, [], []
        for s in range(rng.randint(1, 9)):      # rows share pages
            row = rng.sample(used, rng.randint(0, len(used)))
            held.append(len(row))
            rows.append(row + [rng.choice([-1, 10 ** 6]) for _ in range(columns - len(row))])
            for p in row:
                refs[p] += 1
        for p in used:
            refs[p] = max(refs[p], rng.choice([1, 2]))      # of rows that the call is not given
        moved, movers = ops.compact(refs)
        before = pool.kv.cpu()
        table, new_refs = torch.full((len(rows), columns), -9, dtype=I32, device=DEV), torch.full((n_pages,), -9, dtype=I32, device=DEV)
        got, count = torch.full((2, n_pages), -9, dtype=I32, device=DEV), torch.full((2,), -9, dtype=I32, device=DEV)
        pool.ctx.kv_compact(ints(held), ints(rows), ints(refs), table, new_refs, got, count)
        torch.cuda.synchronize()
        assert count.tolist() == [sum(r > 0 for r in refs), len(movers)]
        assert got.tolist() == [moved, movers + [-1] * (n_pages - len(movers))]
        want = [0] * n_pages
        for p, to in enumerate(moved):
            if to >= 0:
                want[to] = refs[p]
        assert new_refs.tolist() == want
        assert table.tolist() == [[moved[p] for p in r[:h]] + [-1] * (columns - h) for r, h in zip(rows, held)]
        after = before.clone()
        for p in movers:
            after[:, moved[p]] = before[:, p]
        assert torch.equal(pool.kv.cpu(), after)
    pool.close()


def test_pools_of_many_pages(m):
    """More pages than a workgroup looks at in one turn; fork and compact find the same ones as torch does."""
    _, b, _ = m
    n = 70001
    pool = Pool(m, n, heads=1, layers=1)
    g = torch.Generator().manual_seed(5)
    refs = (torch.rand(n, generator=g) < 0.97).to(I32)
    moved, count, table, new_refs = torch.zeros(2, n, dtype=I32, device=DEV), torch.zeros(2, dtype=I32, device=DEV), torch.zeros(1, 4, dtype=I32, device=DEV), torch.zeros(n, dtype=I32, device=DEV)
    last = int(refs.nonzero()[-1])
    before = pool.kv.clone()
    pool.ctx.kv_compact(ints([1]), ints([[last, 0, 0, 0]]), refs.to(DEV), table, new_refs, moved, count)
    torch.cuda.synchronize()
    front = int(refs.sum())
    movers, free = (refs[front:].nonzero()[:, 0] + front), (refs[:front] == 0).nonzero()[:, 0]
    assert count.tolist() == [front, len(movers)] and len(movers) == len(free) > 500
    assert torch.equal(moved[0].cpu()[movers], free.to(I32)) and torch.equal(moved[1].cpu()[:len(movers)], movers.to(I32))
    assert torch.equal(pool.kv[:, free.to(DEV)], before[:, movers.to(DEV)]) and table.tolist() == [[int(free[-1]), -1, -1, -1]]
    assert (new_refs[:front] == 1).all() and (new_refs[front:] == 0).all()
    out = pool.fork([-1] * 60, [], [], [], refs.tolist(), 500, 0, 40)
    assert out["short"] == [0] and sum([r[:32] for r in out["d_new_page_table"]], []) == (refs == 0).nonzero()[:60 * 32, 0].tolist()
    pool.close()


def test_streams_and_graphs(m):
    """A fork and a compaction in one graph, replayed on other parents and counts."""
    _, b, ops = m
    rng = random.Random(8)
    pool = Pool(m, 200)
    n, columns = 6, 14
    cases = [draw(rng, 200, n, 120, columns) for _ in range(4)]
    t = dict(parent=ints([0] * n), length=ints(cases[0][2]), held=ints(cases[0][1]), table=ints(cases[0][0]), refs=ints(cases[0][3]))
    z = lambda *s: torch.zeros(s, dtype=I32, device=DEV)
    out = [dict(d_new_len=z(n), d_new_held=z(n), d_new_page_table=z(n, columns), new_refs=z(200), short=z(1)) for _ in range(2)]
    packed = [(z(n, columns), z(200), z(2, 200), z(2)) for _ in range(2)]

    def run(o, p):
        pool.ctx.kv_fork(t["parent"], t["length"], t["held"], t["table"], t["refs"], room=17, rewrite=16, **o)
        pool.ctx.kv_compact(o["d_new_held"], o["d_new_page_table"], o["new_refs"], *p)

    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        run(out[0], packed[0])
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            run(out[0], packed[0])
    for table, held, length, refs in cases:
        for k, v in (("parent", [rng.randrange(-1, n) for _ in range(n)]), ("length", length), ("held", held), ("table", table), ("refs", refs)):
            t[k].copy_(ints(v))
        start = pool.kv.clone()
        run(out[1], packed[1])
        torch.cuda.synchronize()
        want = pool.kv.clone()
        pool.kv.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool.kv, want) and all(torch.equal(out[0][k], out[1][k]) for k in out[0]) and all(torch.equal(a, c) for a, c in zip(*packed))
        assert out[0]["short"].item() == 0
    pool.close()


def test_refusals(m):
    _, b, _ = m
    pool = Pool(m, 20, max_seqs=4, max_pos=64)
    z = lambda *s: torch.zeros(s, dtype=I32, device=DEV)
    good = dict(parent=z(2), d_len=z(1), d_held=z(1), d_page_table=z(1, 4), refs=z(20), d_new_len=z(2), d_new_held=z(2), d_new_page_table=z(2, 4),
                new_refs=z(20), short=z(1))
    pool.ctx.kv_fork(**good)
    for bad in (dict(parent=z(1)), dict(d_len=None, d_held=z(0)), dict(refs=z(19)), dict(short=z(0)), dict(d_new_page_table=z(2)), dict(new_refs=z(20).cpu()),
                dict(states=[(z(0, 4), z(2, 4))]), dict(states=[(z(1, 4), z(2, 5))]), dict(states=[(z(1, 4), z(2, 4).float())])):
        with pytest.raises(ValueError):
            pool.ctx.kv_fork(**{**good, **bad})
    same = z(20)
    byte = torch.zeros(2, 5, dtype=torch.uint8, device=DEV)
    for bad in (dict(room=-1), dict(room=65), dict(rewrite=-1), dict(rewrite=65), dict(refs=same, new_refs=same), dict(parent=z(5), d_new_len=z(5), d_new_held=z(5), d_new_page_table=z(5, 4)),
                dict(d_len=None), dict(refs=None), dict(parent=None), dict(states=[(byte, byte.clone())]), dict(states=[(same.view(2, 10), same.view(2, 10))]),
                dict(states=[(z(1, 1), z(2, 1))] * 9)):
        with pytest.raises(b.DinferError):
            pool.ctx.kv_fork(**{**good, **bad})
    good = dict(d_held=z(1), d_page_table=z(1, 4), refs=z(20), d_new_page_table=z(1, 4), new_refs=z(20), moved=z(2, 20), count=z(2))
    pool.ctx.kv_compact(**good)
    for bad in (dict(d_page_table=z(4)), dict(moved=z(1, 20)), dict(count=z(1)), dict(d_new_page_table=z(1, 5))):
        with pytest.raises(ValueError):
            pool.ctx.kv_compact(**{**good, **bad})
    for bad in (dict(refs=same, new_refs=same), dict(d_held=None), dict(d_page_table=z(5, 4), d_held=z(5), d_new_page_table=z(5, 4))):
        with pytest.raises(b.DinferError):
            pool.ctx.kv_compact(**{**good, **bad})
    torch.cuda.synchronize()
    pool.close()


def test_pages_beyond_32_bits(m):
    """Pages that lie beyond 4 GiB of a layer are shared, copied and packed as others are."""
    _, b, _ = m
    n = 2 ** 33 // (2 * 2 * 16 * 16 * 128) + 40      # pages of 128 KiB
    pool = Pool(m, 2, dtype="bf16", heads=16, head_dim=128, layers=1)
    pool.close()
    di = m[0]
    cfg = di.configs.scaled(di.model_preset("tiny"), n_layers=1, hidden=64, n_heads=16, head_dim=128, n_experts=1, top_k=1, moe_inter=64, vocab=64, dtype="bf16")
    pool.ctx, pool.n = b.Context(cfg, n, 4, 64, 2048), n
    kv = pool.ctx.kv.view(I32).view(n, -1)
    kv[n - 9:].copy_(torch.randint(0, 2 ** 31 - 1, (9, kv.shape[1]), dtype=I32))
    refs = [0] * (n - 10) + [0] + [1] * 9
    got = pool.fork([0, 0], [20], [2], [[n - 3, n - 1]], [2] * (n - 10) + [0, 2, 2, 2, 2, 2, 2, 1, 2, 1], 5, 0, 3)
    assert got["short"] == [0] and got["d_new_page_table"] == [[n - 3, n - 1, -1], [n - 3, n - 10, -1]]
    assert torch.equal(kv[n - 10], kv[n - 1])
    table, new_refs, moved, count = ints([[0, 0]]), ints([0] * n), torch.zeros(2, n, dtype=I32, device=DEV), ints([0, 0])
    pool.ctx.kv_compact(ints([2]), ints([[n - 1, n - 9]]), ints(refs), table, new_refs, moved, count)
    torch.cuda.synchronize()
    assert count.tolist() == [9, 9] and table.tolist() == [[8, 0]] and torch.equal(kv[:9], kv[n - 9:])
    pool.close()
