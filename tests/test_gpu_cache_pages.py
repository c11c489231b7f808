"""Fork and compact: tables, counts and pages equal those of a page-by-page
implementation, and the cache's operators run together as a serving loop uses
them, also captured into a graph and on another stream."""
import random

import pytest
import torch

import helpers_cache as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _refs(pages, table, extra=()):
    r = torch.zeros(pages, dtype=torch.int32)
    for at in table.flatten().tolist() + list(extra):
        if 0 <= at < pages:
            r[at] += 1
    return r


def _same_pool(cache, pool, pages=None):
    torch.cuda.synchronize()
    for name, got, want in zip(("k", "v", "k_exp", "v_exp"), (cache.k, cache.v, cache.k_exp, cache.v_exp), pool.arrays()):
        assert torch.equal(got.cpu()[:, :pages], want[:, :pages]), name


def _fork(pool, cache, table, lens, refs, parent, grow):
    pages, page = pool.shape[1], pool.shape[3]
    want = H.fork(page, pages, table, lens, refs, parent, grow)
    got = cache.fork(table.to(DEV), lens.to(DEV), refs.to(DEV), parent.to(DEV), None if grow is None else grow.to(DEV))
    H.moved(pool, want[4])
    for name, g, w in zip(("table", "lens", "refs"), got, want):
        assert torch.equal(g.cpu(), w), f"{name}: {g.cpu().tolist()} {w.tolist()}"
    assert int(got[3]) == want[3]
    _same_pool(cache, pool)
    return want


def _i(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_fork_cases():
    pool = H.Pool(1, 3, 20, 2, 16, 64)
    cache = pool.to(DEV)
    table = torch.tensor([[7, 3, 11], [5, -1, -1], [9, 2, -1], [-1, -1, -1]], dtype=torch.int32)
    lens = _i(37, 16, 20, 0)
    refs = _refs(20, table)
    # reorder, drop, fan out, an empty parent, no parent, with pages for what comes
    for parent, grow in (([0, 1, 2, 3], None), ([2, 0], [0, 0]), ([0, 0, 0, 2], [1, 12, 11, 50]), ([3, -1, 4, 1], [5, 5, 0, 0]),
                         ([], None), ([1, 1], [16, 17]), ([2, 2, 2, 2, 2], [0, 13, 0, 0, 29])):
        _fork(pool, cache, table, lens, refs, _i(*parent), None if grow is None else _i(*grow))


def test_fork_held_elsewhere():
    """A page that someone else holds too is never appended to; one that is given back can be taken at once."""
    pool = H.Pool(2, 1, 8, 1, 32, 128)
    cache = pool.to(DEV)
    table = torch.tensor([[6, 1, 4], [0, 2, -1]], dtype=torch.int32)
    lens = _i(70, 33)
    for extra in ([], [4], [6, 2], [4, 4, 2]):
        _fork(pool, cache, table, lens, _refs(8, table, extra), _i(0, 1), _i(0, 40))
        _fork(pool, cache, table, lens, _refs(8, table, extra), _i(1, 1), _i(64, 0))


@pytest.mark.parametrize("width", [2, 3000])
def test_fork_shared_tails(width):
    """Rows that share a partly filled page: every child copies it, and it is not taken meanwhile."""
    pool = H.Pool(4, 2, 12, 2, 16, 128)
    cache = pool.to(DEV)
    table = torch.full((4, width), -1, dtype=torch.int32)
    table[:, :2] = torch.tensor([[5, 1], [4, 1], [3, 2], [6, 2]])
    for parent in (_i(2, 3, 0, 1), _i(2, 2, 3, 3, 1, 0, 0), _i(3, 0)):
        _fork(pool, cache, table, _i(20, 25, 17, 31), _refs(12, table), parent, torch.zeros_like(parent))
        _fork(pool, cache, table, _i(20, 25, 17, 31), _refs(12, table, [1]), parent, None)


def test_fork_runs_out():
    """Too few pages, or a table too narrow: counted, -1, and nothing else suffers."""
    pool = H.Pool(3, 2, 6, 1, 16, 64)
    cache = pool.to(DEV)
    table = torch.tensor([[0, 1, -1], [3, -1, -1]], dtype=torch.int32)
    refs = _refs(6, table, [5])
    _fork(pool, cache, table, _i(20, 7), refs, _i(0, 0, 0, 1, 1), _i(0, 0, 0, 0, 0))
    _fork(pool, cache, table, _i(20, 7), refs, _i(1, 0), _i(100, 3))
    _fork(pool, cache, table, _i(20, 7), refs, _i(1, 0), _i(2 ** 31 - 1, 2 ** 31 - 1))
    _fork(pool, cache, table, _i(2 ** 31 - 1, -5), refs, _i(0, 1), _i(-3, 1))


@pytest.mark.parametrize("seed", range(10))
def test_fork_random(seed):
    """Small batches (one workgroup keeps the books) and, from seed 6 on, wide tables (the grid does)."""
    r = random.Random(seed)
    page, pages = r.choice([16, 64]), r.choice([40, 1100, 2500])
    B = r.choice([3, 17, 60])
    lens = [r.randint(0, 5 * page) for _ in range(B)]
    pool = H.Pool(seed, 1, pages + 6 * B, 1, page, 64)
    cache = pool.to(DEV)
    table = pool.tables(lens, width=7 if seed < 6 else 3000)
    extra = [r.randrange(pages) for _ in range(r.randint(0, 30))]
    parent = [r.randint(-1, B) for _ in range(r.choice([2, B, 2 * B]))]
    grow = [r.choice([0, 1, page, 3 * page]) for _ in parent]
    _fork(pool, cache, table, _i(*lens), _refs(pool.shape[1], table, extra), _i(*parent), _i(*grow))


def test_fork_in_place_counts():
    """refs_out may be refs_in; table and lengths may not overlap their inputs."""
    import paper_2602_02071_amd as baps
    pool = H.Pool(4, 1, 9, 1, 16, 64)
    cache = pool.to(DEV)
    table, lens = torch.tensor([[1, 8], [4, -1]], dtype=torch.int32), _i(30, 16)
    refs = _refs(9, table)
    want = H.fork(16, 9, table, lens, refs, _i(0, 0, 1), None)
    t, n, r, par = table.to(DEV), lens.to(DEV), refs.to(DEV), _i(0, 0, 1).to(DEV)
    out, out_n, miss = torch.empty((3, 2), dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV), r.new_empty(1)
    nbytes = baps.baps_cache_pages_workspace(0, 3)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    baps.baps_cache_fork(cache.c, t, n, r, 2, par, None, 3, 2, out, out_n, r, miss, ws, nbytes)
    assert torch.equal(out.cpu(), want[0]) and torch.equal(r.cpu(), want[2]) and int(miss) == 0
    H.moved(pool, want[4])
    _same_pool(cache, pool)
    with pytest.raises(baps.BapsError):
        baps.baps_cache_fork(cache.c, t, n, r, 2, par, None, 2, 2, t, out_n, r, miss, ws, nbytes)


@pytest.mark.parametrize("pages,live", [(1, 0.5), (5, 0.5), (64, 0.3), (1024, 0.7), (1025, 0.5), (3001, 0.05), (3001, 0.97),
                                        (4096, 1.0), (2048, 0.0)])
def test_compact(pages, live):
    pool = H.Pool(pages, 2, pages, 1, 16, 64)
    cache = pool.to(DEV)
    refs = (torch.rand(pages, generator=pool.g) < live).to(torch.int32) * torch.randint(1, 4, (pages,), generator=pool.g, dtype=torch.int32)
    table = torch.randint(-2, pages + 2, (5, 13), generator=pool.g, dtype=torch.int32)
    want = H.compact(pages, table, refs)
    got = cache.compact(table.to(DEV), refs.to(DEV))
    for name, g, w in zip(("table", "refs", "remap"), got, want):
        assert torch.equal(g.cpu(), w), name
    assert int(got[3]) == want[3]
    H.moved(pool, want[4])
    _same_pool(cache, pool, want[3])


def test_compact_in_place():
    import paper_2602_02071_amd as baps
    pool = H.Pool(9, 1, 300, 2, 32, 128)
    cache = pool.to(DEV)
    refs = torch.randint(0, 2, (300,), generator=pool.g, dtype=torch.int32)
    table = torch.randint(-1, 300, (4, 50), generator=pool.g, dtype=torch.int32)
    want = H.compact(300, table, refs)
    t, r = table.to(DEV), refs.to(DEV)
    remap, n = torch.empty_like(r), r.new_empty(1)
    nbytes = baps.baps_cache_pages_workspace(300, 0)
    baps.baps_cache_compact(cache.c, t, t.numel(), r, t, r, remap, n, torch.empty(nbytes, dtype=torch.uint8, device=DEV), nbytes)
    assert torch.equal(t.cpu(), want[0]) and torch.equal(r.cpu(), want[1]) and torch.equal(remap.cpu(), want[2])
    H.moved(pool, want[4])
    _same_pool(cache, pool, want[3])


# ------------------------------------------------------------------ together
class _Mirror:
    """The cache's state on the CPU, moved by the plain implementations."""

    def __init__(self, seed, layers, pages, Hkv, page, D):
        self.pool = H.Pool(seed, layers, pages, Hkv, page, D)
        self.table, self.lens, self.refs = torch.zeros((0, 12), dtype=torch.int32), _i(), torch.zeros(pages, dtype=torch.int32)

    def fork(self, parent, grow):
        layers, pages, Hkv, page, D = self.pool.shape
        t, n, r, miss, copies = H.fork(page, pages, self.table, self.lens, self.refs, parent, grow)
        assert miss == 0
        H.moved(self.pool, copies)
        self.table, self.lens, self.refs = t, n, r

    def compact(self):
        t, r, remap, n, moves = H.compact(self.pool.shape[1], self.table, self.refs)
        H.moved(self.pool, moves)
        self.table, self.refs = t, r


@pytest.mark.parametrize("stream", [False, True])
def test_serving_loop(stream):
    """Prompts, decode steps, beams that fork and end, a compaction, more decode: every output against 64 bits."""
    layers, pages, Hkv, page, D, Hq, W, S = 2, 60, 2, 16, 64, 4, 40, 3
    m = _Mirror(31, layers, pages, Hkv, page, D)
    side = torch.cuda.Stream() if stream else torch.cuda.current_stream()
    with torch.cuda.stream(side):
        cache = m.pool.to(DEV)
        table, lens, refs = (x.to(DEV) for x in (m.table, m.lens, m.refs))
        g = m.pool.g
        plan = [([-1, -1, -1], [50, 7, 33]), ([0, 1, 2], [1] * 3), ([0, 0, 2, 0], [1] * 4), ([3, 1, 1, 2], [4] * 4), "compact",
                ([0, 1, 2, 3, 3, 3], [1] * 6), ([5, 0], [70, 70])]
        for step in plan:
            if step == "compact":
                m.compact()
                table, refs, remap, live = cache.compact(table, refs)
                continue
            parent, new = step
            m.fork(_i(*parent), _i(*new))
            table, lens, refs, missing = cache.fork(table, lens, refs, _i(*parent).to(DEV), _i(*new).to(DEV))
            lens = lens + _i(*new).to(DEV)
            m.lens = m.lens + _i(*new)
            cu = [sum(new[:i]) for i in range(len(new) + 1)]
            for layer in range(layers):
                q, k, v = (torch.randn((sum(new), h, D), generator=g).to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
                H.append(m.pool, layer, k, v, cu, m.lens, m.table)
                cache.append(layer, k.to(DEV), v.to(DEV), H.ints(cu, DEV), lens, table, max(new))
                o, lse = cache.attention(layer, q.to(DEV), H.ints(cu, DEV), lens, table, max(new), int(m.lens.max()), W, S)
                ref = []
                for b, n in enumerate(m.lens.tolist()):
                    kk, vv, ok = H.sequence_kv(m.pool, layer, m.table[b], n)
                    ref.append(H.attend(q[cu[b]:cu[b + 1]], kk, vv, range(n - new[b], n), W, S))
                few = max(new) * (Hq // Hkv) <= 64
                H.check(o, lse, [torch.cat(x) for x in zip(*ref)], 130, D, 2.0 ** -16 if few else 2.0 ** -8, f"{step} {layer}")
            assert torch.equal(table.cpu(), m.table) and torch.equal(refs.cpu(), m.refs) and int(missing) == 0


def test_captured_step():
    """A decode step captured once and replayed: it follows what tables, lengths and inputs hold at each replay."""
    pool = H.Pool(41, 1, 40, 2, 16, 128)
    eager, captured = pool.to(DEV), pool.to(DEV)
    lens0 = [30, 5, 700 // 8]
    table = pool.tables([120, 120, 120]).to(DEV)
    q, k, v = (torch.zeros((3, h, 128), dtype=torch.bfloat16, device=DEV) for h in (8, 2, 2))
    lens, cu = H.ints(lens0, DEV), H.ints([0, 1, 2, 3], DEV)
    parent = H.ints([0, 1, 2], DEV)
    refs = _refs(40, table.cpu()).to(DEV)

    def step(cache):
        cache.append(0, k, v, cu, lens, table, 1)
        # (a length bound that splits the keys: the workspace is part of the graph)
        o, lse = cache.attention(0, q, cu, lens, table, 1, 4000, 64, 4)
        return o, lse, cache.fork(table, lens, refs, parent)[0]

    step(captured)
    captured.k.copy_(eager.k), captured.v.copy_(eager.v), captured.k_exp.copy_(eager.k_exp), captured.v_exp.copy_(eager.v_exp)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(captured)
    for i in range(4):
        g = torch.Generator().manual_seed(i)
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g).to(torch.bfloat16))
        lens += 1
        want = step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), i
        for a, b in ((captured.k, eager.k), (captured.v, eager.v), (captured.k_exp, eager.k_exp), (captured.v_exp, eager.v_exp)):
            assert torch.equal(a, b), i
