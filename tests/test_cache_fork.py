"""Forking and compacting the pages of a cache against tables kept by plain loops, and the refusals (on the CPU)."""
import ctypes

import numpy as np
import pytest

from paper_2602_21788_amd import binding as B


# ---- the definitions, one sequence after the other --------------------------------------------------------------------------------------------
def fork(pages, lens, parent, news, n_pages, P, busy):
    """pages [n][m], lens [n]: tables as numpy.  Returns new tables, lengths, counts, and the copies (from, to, tokens)."""
    m = pages.shape[1]
    valid = lambda p: 0 <= p < n_pages
    clipped = [min(max(int(n), 0), m * P) for n in lens]
    old = [[int(p) if valid(p) else -1 for p in row[: -(-n // P)]] for row, n in zip(pages, clipped)]
    held = {p for t in old for p in t if p >= 0} | {int(p) for p in np.flatnonzero(busy)}
    free = [p for p in range(n_pages) if p not in held]
    tables, before, after, reads, writers = [], [], [], {int(p) for p in np.flatnonzero(busy)}, {}
    for i, (p, new) in enumerate(zip(parent, news)):
        there = 0 <= p < len(old)
        t, n = (list(old[p]), clipped[p]) if there else ([], 0)
        grown = min(n + max(int(new), 0), m * P)
        written = n // P if grown > n and n % P else -1
        for j, page in enumerate(t):
            if page >= 0 and j == written:
                writers.setdefault(page, []).append(i)
            elif page >= 0:
                reads.add(page)
        tables.append(t)
        before.append(n)
        after.append(grown)
    copies, lacking, taken = [], 0, 0

    def fresh():
        nonlocal lacking, taken
        if taken < len(free):
            taken += 1
            return free[taken - 1]
        lacking += 1
        return -1

    for i, t in enumerate(tables):
        if after[i] > before[i] and before[i] % P and t[before[i] // P] >= 0:
            page = t[before[i] // P]
            if page in reads or writers[page][0] != i:
                t[-1] = fresh()
                if t[-1] >= 0:
                    copies.append((page, t[-1], before[i] % P))
        while len(t) * P < after[i]:
            t.append(fresh())
    holds = {p for t in tables for p in t if p >= 0} | {int(p) for p in np.flatnonzero(busy)}
    table = np.array([t + [-1] * (m - len(t)) for t in tables], np.int32).reshape(len(tables), m)
    return table, np.array(after, np.int32), [taken, lacking, n_pages - len(holds)], copies


def compact(pages, lens, n_pages, P, busy):
    m = pages.shape[1]
    held = [[int(p) if 0 <= p < n_pages else -1 for p in row[: -(-min(max(int(n), 0), m * P) // P)]] for row, n in zip(pages, lens)]
    in_use = {p for t in held for p in t if p >= 0}
    moving = sorted(p for p in in_use if not busy[p])
    low = [p for p in range(n_pages) if not busy[p]][: len(moving)]
    holes, to = [p for p in low if p not in in_use], {}
    for p in moving:
        if p not in set(low):
            to[p] = holes[len(to)]
    end = max([-1] + low + [int(p) for p in np.flatnonzero(busy)]) + 1
    table = np.array([[to.get(p, p) for p in t] + [-1] * (m - len(t)) for t in held], np.int32).reshape(len(held), m)
    return table, [len(to), len(in_use), end], [(a, b, P) for a, b in to.items()]


def test_definitions():
    """Three beams of a sequence of 20 tokens in pages of 16: the lowest goes on in its page, the others copy 4 tokens; who only reads keeps everybody from writing."""
    pages, busy = np.array([[3, 1, -1], [3, 0, -1]], np.int32), np.zeros(8, np.uint8)
    t, n, c, copies = fork(pages, [20, 16], [0, 0, 0, 1, 5], [1, 1, 13, 1, 2], 8, 16, busy)
    assert t.tolist() == [[3, 1, -1], [3, 0, -1], [3, 2, 4], [3, 5, -1], [6, -1, -1]] and n.tolist() == [21, 21, 33, 17, 2]
    assert copies == [(1, 0, 4), (1, 2, 4)] and c == [5, 0, 1]
    t, n, c, copies = fork(pages, [20, 16], [0, 0], [0, 1], 8, 16, busy)
    assert t.tolist() == [[3, 1, -1], [3, 0, -1]] and copies == [(1, 0, 4)] and c == [1, 0, 5]
    t, c, copies = compact(np.array([[6, 2], [6, 7]], np.int32), [32, 20], 9, 16, np.array([0, 1, 0, 0, 0, 0, 0, 0, 1]))
    assert t.tolist() == [[0, 2], [0, 3]] and c == [2, 3, 9] and copies == [(6, 0, 16), (7, 3, 16)]


# ---- CPU ------------------------------------------------------------------------------------------------------------------------------------
class Call:
    """Calls with addresses that nobody looks at: every one below fails first."""
    def __init__(self, **kw):
        f = self.f = 0x10000
        self.c = B.Cache.__new__(B.Cache)
        for name, v in dict(_k=f, _v=f, _k_scale=f, _v_scale=f, _weight=None, n_pages=9, hkv=4, head_dim=128, page_tokens=64, format=0).items():
            setattr(self.c, name, kw.pop(name, v))
        self.kw = kw

    def a(self, name, v):
        return self.kw.get(name, v)

    def ref(self):
        return None if self.kw.get("no_cache") else ctypes.byref(self.c)

    def fork(self):
        a, f = self.a, self.f
        return B.lib().fcp_cache_fork(self.ref(), a("pages", f), a("kv_len", f), a("n_seqs", 2), a("max_pages", 3), a("parent", f), a("news", f), a("n_new", 4), a("busy", None),
                                      a("new_pages", f + 64), a("new_len", f + 128), a("counts", f + 256), a("scratch", f), a("bytes", 1 << 40), None)

    def compact(self):
        a, f = self.a, self.f
        return B.lib().fcp_cache_compact(self.ref(), a("pages", f), a("kv_len", f), a("n_seqs", 2), a("max_pages", 3), a("busy", None), a("new_pages", f), a("counts", f + 256),
                                         a("scratch", f), a("bytes", 1 << 40), None)


def test_refusals_come_before_any_device_work():
    bad, no, full = B.FCP_ERR_INVALID_ARG, B.FCP_ERR_UNSUPPORTED, B.FCP_ERR_CAPACITY
    for op in ("fork", "compact"):
        call = lambda **kw: getattr(Call(**kw), op)()
        for kw in (dict(no_cache=True), dict(_k=None), dict(_v_scale=None), dict(n_pages=0), dict(_k=0x10008), dict(n_seqs=-1), dict(max_pages=-1), dict(pages=None), dict(kv_len=None),
                   dict(new_pages=None), dict(counts=None), dict(scratch=None), dict(scratch=0x10080)):
            assert call(**kw) == bad, (op, kw)
            assert f"fcp_cache_{op}".encode() in B.lib().fcp_last_error()
        for kw in (dict(head_dim=96), dict(page_tokens=48), dict(format=2), dict(hkv=5000), dict(n_seqs=(1 << 20) + 1), dict(max_pages=1 << 25), dict(n_seqs=1 << 20, max_pages=1 << 13)):
            assert call(**kw) == no, (op, kw)
        which = B.FCP_SCRATCH_CACHE_FORK if op == "fork" else B.FCP_SCRATCH_CACHE_COMPACT
        need = B.fcp_cache_scratch_bytes(which, Call().c, 4 if op == "fork" else 2, 3)
        assert call(bytes=need - 1) == full
    for kw in (dict(n_new=-1), dict(parent=None), dict(news=None), dict(new_len=None), dict(new_pages=0x10000), dict(new_len=0x10000)):
        assert Call(**kw).fork() == bad, kw
    for kw in (dict(n_new=(1 << 20) + 1), dict(n_new=1 << 20, hkv=16), dict(n_new=1 << 20, max_pages=1 << 12)):
        assert Call(**kw).fork() == no, kw


def test_scratch_sizes():
    c = Call().c
    for which in (B.FCP_SCRATCH_CACHE_FORK, B.FCP_SCRATCH_CACHE_COMPACT):
        assert B.fcp_cache_scratch_bytes(which, c, 0, 0) > 0
        with pytest.raises(B.FcpError):
            B.fcp_cache_scratch_bytes(which, c, -1, 3)
        with pytest.raises(B.FcpError):
            B.fcp_cache_scratch_bytes(which, c, 1 << 20, 1 << 13)
    assert B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_FORK, c, 1000, 3) > B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_FORK, c, 1, 3)
    c.n_pages = 100000
    assert B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_COMPACT, c, 1, 3) > 100000 * 16


# ---- GPU ------------------------------------------------------------------------------------------------------------------------------------
class Pool:
    """A cache of random bytes, scales and weights, and the same on the host."""
    def __init__(self, rng, n_pages, P, hkv=2, D=64, fmt="int8", weight=True):
        import torch
        self.P, self.n = P, n_pages
        dt = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
        raw = lambda *s: rng.integers(0, 256, s, dtype=np.uint8)
        self.host = {"k": raw(n_pages, hkv, P, D), "v": raw(n_pages, hkv, P // 16, D, 16), "k_scale": rng.random((n_pages, hkv), np.float32),
                     "v_scale": rng.random((n_pages, hkv), np.float32), "weight": rng.random((n_pages, hkv, P), np.float32)}
        d = {k: torch.from_numpy(v.copy()).cuda() for k, v in self.host.items()}
        self.cache = B.Cache(d["k"].view(dt), d["v"].view(dt), d["k_scale"], d["v_scale"], d["weight"] if weight else None)
        self.dev, self.weight = d, weight

    def move(self, copies):
        """Done on the host; the sources are nobody's target."""
        for a, b, n in copies:
            for name, k in (("k", n), ("v", -(-n // 16)), ("weight", n if self.weight else 0)):
                self.host[name][b, :, :k] = self.host[name][a, :, :k]
            for name in ("k_scale", "v_scale"):
                self.host[name][b] = self.host[name][a]

    def same(self):
        for k, v in self.host.items():
            assert np.array_equal(self.dev[k].cpu().numpy(), v), k


def _dev(a, dtype=np.int32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def _fork(pool, pages, lens, parent, news, busy=None, stream=None):
    import torch
    n, m = len(parent), pages.shape[1]
    table, new_len, counts = (torch.full(s, 99, dtype=torch.int32, device="cuda") for s in ((n + 1, m), (n + 1,), (4,)))
    scratch = torch.full((B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_FORK, pool.cache, n, m),), 255, dtype=torch.uint8, device="cuda")
    B.fcp_cache_fork(pool.cache, _dev(pages), _dev(lens), _dev(parent), _dev(news), table[:n], new_len[:n], counts, scratch, None if busy is None else _dev(busy, np.uint8), stream)
    torch.cuda.synchronize()
    want = fork(pages, lens, parent, news, pool.n, pool.P, np.zeros(pool.n, np.uint8) if busy is None else busy)
    assert np.array_equal(table[:n].cpu().numpy(), want[0])
    assert np.array_equal(new_len[:n].cpu().numpy(), want[1]) and counts.tolist() == want[2] + [99] and (table[n] == 99).all() and new_len[n] == 99
    pool.move(want[3])
    pool.same()
    return want


def _compact(pool, pages, lens, busy=None, in_place=False):
    import torch
    n, m = pages.shape
    old = _dev(pages)
    table = old if in_place else torch.full((n, m), 99, dtype=torch.int32, device="cuda")
    counts = torch.full((3,), 99, dtype=torch.int32, device="cuda")
    scratch = torch.full((B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_COMPACT, pool.cache, n, m),), 255, dtype=torch.uint8, device="cuda")
    B.fcp_cache_compact(pool.cache, old, _dev(lens), table, counts, scratch, None if busy is None else _dev(busy, np.uint8))
    torch.cuda.synchronize()
    want = compact(pages, lens, pool.n, pool.P, np.zeros(pool.n, np.uint8) if busy is None else busy)
    assert np.array_equal(table.cpu().numpy(), want[0]) and counts.tolist() == want[1]
    pool.move(want[2])
    pool.same()
    return want


def _padded(pages, lens, large):
    """large: thousands of sequences without tokens behind the others, so that the call is worked as large ones are."""
    if not large:
        return pages, lens
    return np.concatenate([pages, np.full((4100, pages.shape[1]), -1, np.int32)]), np.concatenate([lens, np.zeros(4100, np.int32)])


def _tables(rng, n, m, n_pages, P, busy):
    """Sequences of any length, some with a common beginning."""
    lens = rng.integers(0, m * P + 1, n)
    lens[rng.random(n) < 0.3] //= 8
    lens[rng.random(n) < 0.2] = lens[rng.random(n) < 0.2].sum() // max(n, 1) // P * P
    order = [int(p) for p in rng.permutation(n_pages) if not busy[p]]
    pages = np.full((n, m), -1, np.int32)
    for i in range(n):
        shared = 0
        if i and rng.random() < 0.5:
            j = int(rng.integers(0, i))
            shared = int(rng.integers(0, min(lens[i], lens[j]) // P + 1))
            pages[i, :shared] = pages[j, :shared]
        for k in range(shared, -(-int(lens[i]) // P)):
            pages[i, k] = order.pop() if order else -1
    return pages, lens.astype(np.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("P, hkv, D, fmt, weight", [(16, 2, 64, "int8", True), (32, 3, 128, "e4m3", False), (64, 1, 128, "int8", True), (128, 5, 64, "e4m3", True)])
@pytest.mark.parametrize("n, n_new, m, n_pages", [(1, 8, 4, 40), (8, 8, 5, 90), (70, 130, 3, 700), (5, 3, 130, 900), (2, 9, 600, 1200), (3, 0, 2, 9), (0, 4, 2, 9)])
def test_fork(P, hkv, D, fmt, weight, n, n_new, m, n_pages, large):
    rng = np.random.default_rng(n * 1000 + n_new + P)
    busy = (rng.random(n_pages) < 0.1).astype(np.uint8)
    pool = Pool(rng, n_pages, P, hkv, D, fmt, weight)
    pages, lens = _padded(*_tables(rng, n, m, n_pages, P, busy), large)
    parent = rng.integers(-1, n + 1, n_new)                  # (some of nobody)
    for news in (np.ones(n_new), np.zeros(n_new), rng.integers(-1, 2 * P, n_new)):
        _fork(pool, pages, lens, parent, news.astype(np.int32), busy)
    _fork(pool, pages, lens, parent, np.ones(n_new, np.int32))          # (pages that were busy are free)


@pytest.mark.gpu
@pytest.mark.parametrize("large", [False, True])
def test_fork_keeps_a_page_that_others_read_or_hold(large):
    """A sequence goes on in a page of which another one has more tokens, of which another one reads as many, that is busy, that a table names twice."""
    rng = np.random.default_rng(7)
    pool = Pool(rng, 30, 32)
    pages = np.array([[4, 9, -1], [4, 9, 2], [4, 9, -1], [7, 7, -1], [8, -1, -1]], np.int32)
    lens = np.array([50, 70, 50, 40, 3], np.int32)
    pages, lens = _padded(pages, lens, large)
    busy = np.zeros(30, np.uint8)
    busy[8] = 1
    for parent, news in (([0, 1], [1, 1]), ([0, 2], [1, 0]), ([2, 0, 0], [5, 1, 40]), ([3, 3], [1, 1]), ([4], [1]), ([4, 4], [0, 0]), ([1, 1, 0, 2, 3, 4], [1] * 6)):
        for b in (None, busy):
            _fork(pool, pages, lens, np.array(parent), np.array(news), b)


@pytest.mark.gpu
@pytest.mark.parametrize("large", [False, True])
def test_fork_with_too_few_pages_and_entries_that_are_no_page(large):
    rng = np.random.default_rng(8)
    pool = Pool(rng, 6, 16)
    pages = np.array([[0, 1, -1, -1], [2, 99, 3, -1], [-7, -1, -1, -1]], np.int32)
    for lens in ([20, 40, 10], [32, 48, 16], [1000, 17, -3], [0, 0, 0]):
        for parent in ([0, 0, 0, 0], [1, 1, 0], [2, 2, 2], [0, 1, 2, 3, -1]):
            for new in (1, 20, 1 << 30):
                _fork(pool, *_padded(pages, np.array(lens, np.int32), large), np.array(parent), np.full(len(parent), new))


@pytest.mark.gpu
@pytest.mark.parametrize("n, m, n_pages, n_new", [(2500, 9, 70001, 3001), (4100, 3, 30011, 1000), (300, 4, 20000, 8200), (600, 300, 262160, 20)])
def test_fork_many(n, m, n_pages, n_new):
    """More sequences and pages than a block looks at once; more than are worked by one block."""
    rng = np.random.default_rng(9)
    pool = Pool(rng, n_pages, 16, hkv=1)
    pages, lens = _tables(rng, n, m, n_pages, 16, np.zeros(n_pages))
    parent = rng.integers(0, n, n_new)
    w = _fork(pool, pages, lens, parent, rng.integers(0, 40, n_new))
    _compact(pool, w[0], w[1])


@pytest.mark.gpu
@pytest.mark.parametrize("n, m, n_pages, n_new", [(300, 9, 70001, 1000), (20, 30, 262144, 1024), (1000, 30, 40000, 1024), (64, 30, 65569, 700)])
def test_one_block_over_many_pages(n, m, n_pages, n_new):
    """Pools of more pages than a block's threads look at once, where one block marks and plans; more fresh pages than LDS lists; some busy."""
    rng = np.random.default_rng(n)
    pool = Pool(rng, n_pages, 16, hkv=1)
    busy = (rng.random(n_pages) < 0.3).astype(np.uint8)
    pages, lens = _tables(rng, n, m, n_pages, 16, busy)
    for high in (20, 150):
        w = _fork(pool, pages, lens, rng.integers(-1, n, n_new), rng.integers(0, high, n_new), busy)
        _compact(pool, w[0], w[1], busy)


@pytest.mark.gpu
def test_every_page_of_a_block_held():
    """32768 pages, all of them held, and read by sequences that go on; then all but one, which moves."""
    rng = np.random.default_rng(1)
    pool = Pool(rng, 32768, 16, hkv=1)
    pages, lens = rng.permutation(32768).astype(np.int32).reshape(1024, 32), np.full(1024, 512, np.int32)
    w = _fork(pool, pages, lens, np.arange(1024), np.zeros(1024, np.int32))
    assert w[2] == [0, 0, 0]
    assert _compact(pool, pages, lens)[1] == [0, 32768, 32768]
    at = tuple(np.argwhere(pages == 5)[0])
    pages[at] = -1
    assert _compact(pool, pages, lens)[1] == [1, 32767, 32767]
    w = _fork(pool, pages, lens - 3, np.arange(1024), np.ones(1024, np.int32))
    assert w[2] == [0, 0, 1]


@pytest.mark.gpu
def test_steps_one_after_the_other():
    """A prompt, its beams, and then every step's tables out of those before; compacted in between."""
    rng = np.random.default_rng(10)
    pool = Pool(rng, 120, 16)
    pages = np.full((2, 8), -1, np.int32)
    pages[0, :3], pages[1, :2] = (50, 40, 30), (20, 10)
    lens = np.array([41, 32], np.int32)
    parent, news = np.repeat([0, 1], 4), np.ones(8, np.int32)
    for step in range(40):
        w = _fork(pool, pages, lens, parent, news)
        pages, lens = w[0], w[1]
        parent = np.concatenate([rng.integers(0, 4, 4), rng.integers(4, 8, 4)])
        if step % 9 == 5:
            pages = _compact(pool, pages, lens)[0]
        assert w[2][1] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("P, hkv, D, fmt, weight", [(16, 2, 64, "int8", True), (128, 3, 128, "e4m3", False)])
@pytest.mark.parametrize("n, m, n_pages, share", [(1, 1, 1, 0), (1, 5, 33, 0.2), (9, 6, 64, 0.0), (40, 7, 900, 0.3), (0, 3, 40, 0.5), (3, 0, 9, 0.5), (300, 5, 4000, 0.02)])
def test_compact(P, hkv, D, fmt, weight, n, m, n_pages, share, large):
    rng = np.random.default_rng(n + n_pages)
    busy = (rng.random(n_pages) < share).astype(np.uint8)
    pool = Pool(rng, n_pages, P, hkv, D, fmt, weight)
    pages, lens = _tables(rng, n, m, n_pages, P, busy)
    if n > 5:
        busy[pages[pages >= 0][:3]] = 1                      # pages in use that stay
        pages[2, 0], lens[3] = 10 ** 6, -1
    pages, lens = _padded(pages, lens, large)
    w = _compact(pool, pages, lens, busy)
    _compact(pool, w[0], lens, busy, in_place=True)          # (nothing moves any more)
    if not busy.any():
        assert len(w[2]) == w[1][0] and w[1][2] == w[1][1]
    _compact(pool, w[0], lens, in_place=True)


@pytest.mark.gpu
def test_graphs_of_steps_replay():
    """A step to and one fro captured in a graph: every replay continues what the replay before left, other work between."""
    import torch
    rng = np.random.default_rng(11)
    pool = Pool(rng, 200, 16)
    n, m, P = 6, 12, 16
    pages = np.full((n, m), -1, np.int32)
    pages[:, :2] = rng.permutation(200)[: 2 * n].reshape(n, 2)
    lens = np.full(n, 20, np.int32)
    a, b = [_dev(pages), _dev(lens)], [torch.empty(n, m, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")]
    parent, news, counts = _dev(np.zeros(n)), _dev(np.ones(n)), torch.empty(3, dtype=torch.int32, device="cuda")
    scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_FORK, pool.cache, n, m), dtype=torch.uint8, device="cuda")
    there, back = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    for g, x, y in ((there, a, b), (back, b, a)):
        with torch.cuda.graph(g):
            B.fcp_cache_fork(pool.cache, *x, parent, news, *y, counts, scratch)
    for step in range(20):
        p = rng.integers(0, n, n)
        parent.copy_(_dev(p))
        (there, back)[step % 2].replay()
        other = torch.randn(1 << 16, device="cuda").sum()
        x = (b, a)[step % 2]
        pages, lens, c, copies = fork(pages, lens, p, np.ones(n, np.int32), 200, P, np.zeros(200))
        assert np.array_equal(x[0].cpu().numpy(), pages) and np.array_equal(x[1].cpu().numpy(), lens) and counts.tolist() == c and bool(torch.isfinite(other))
        pool.move(copies)
        pool.same()


@pytest.mark.gpu
def test_binding_refuses_tensors_of_other_types_and_sizes():
    import torch
    pool = Pool(np.random.default_rng(12), 9, 16)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    w = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    for bad in (lambda: B.fcp_cache_fork(pool.cache, i(2, 3), i(2), i(4), i(4), i(4, 2), i(4), i(3), w), lambda: B.fcp_cache_fork(pool.cache, i(2, 3), i(2), i(3), i(4), i(4, 3), i(4), i(3), w),
                lambda: B.fcp_cache_fork(pool.cache, i(2, 3), i(2), i(4), i(4), i(4, 3), i(3), i(3), w), lambda: B.fcp_cache_fork(pool.cache, i(2, 3), i(1), i(4), i(4), i(4, 3), i(4), i(3), w),
                lambda: B.fcp_cache_fork(pool.cache, i(2, 3), i(2), i(4), i(4), i(4, 3), i(4), i(2), w), lambda: B.fcp_cache_fork(pool.cache, i(2, 3).long(), i(2), i(4), i(4), i(4, 3), i(4), i(3), w),
                lambda: B.fcp_cache_fork(pool.cache, i(2, 3), i(2), i(4), i(4), i(4, 3), i(4), i(3), w, busy=i(9)), lambda: B.fcp_cache_compact(pool.cache, i(2, 3), i(2), i(2, 4), i(3), w),
                lambda: B.fcp_cache_compact(pool.cache, i(2, 3), i(2), i(2, 3), i(3), w, busy=w[:8])):
        with pytest.raises(ValueError):
            bad()
