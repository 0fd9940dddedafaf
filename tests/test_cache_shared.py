"""Attention over the cache behind a common beginning against attention over every sequence's whole table, in 64 bits (tests/cache_ref.py), and the refusals (on the CPU)."""
import ctypes

import numpy as np
import pytest

import cache_ref as R
from paper_2602_21788_amd import binding as B
from test_cache import check_attn, dev, dev_bf16

FORMATS = ["e4m3", "int8"]


# ---- CPU ------------------------------------------------------------------------------------------------------------------------------------
def _call(**kw):
    """A call with addresses that nobody looks at: every one below fails first, or has nothing to do."""
    f = 0x10000
    c = B.Cache.__new__(B.Cache)
    for name, v in dict(_k=f, _v=f, _k_scale=f, _v_scale=f, _weight=None, n_pages=9, hkv=4, head_dim=128, page_tokens=64, format=0).items():
        setattr(c, name, kw.pop(name, v))
    a = lambda name, v: kw.get(name, v)
    return B.lib().fcp_cache_attn_shared(None if a("no_cache", 0) else ctypes.byref(c), a("q", f), a("q_row", 2048), a("tq", 4), a("hq", 16), a("cu", f), a("kv_len", f), a("pages", f),
                                         a("n_seqs", 4), a("max_pages", 3), a("groups", f), a("shared", f), a("n_groups", 2), a("scale", 0.1), a("o", f), a("lse", f), a("scratch", f),
                                         a("bytes", 1 << 40), None)


def test_refusals_come_before_any_device_work():
    bad, no, full = B.FCP_ERR_INVALID_ARG, B.FCP_ERR_UNSUPPORTED, B.FCP_ERR_CAPACITY
    for kw in (dict(no_cache=1), dict(_v=None), dict(n_pages=0), dict(_k=0x10008), dict(n_seqs=-1), dict(max_pages=-1), dict(tq=-1), dict(cu=None), dict(kv_len=None), dict(pages=None),
               dict(scale=0.0), dict(scale=float("nan")), dict(scale=2.0 ** -33), dict(n_groups=-1), dict(n_groups=5), dict(groups=None), dict(shared=None), dict(q=None), dict(q_row=2040),
               dict(q_row=2052), dict(q=0x10008), dict(o=None), dict(lse=None), dict(o=0x10008), dict(lse=0x10002), dict(scratch=None), dict(scratch=0x10010)):
        assert _call(**kw) == bad, kw
        assert b"fcp_cache_attn_shared" in B.lib().fcp_last_error()
    for kw in (dict(hq=6), dict(hq=0), dict(head_dim=96), dict(page_tokens=48), dict(format=2), dict(n_seqs=(1 << 20) + 1), dict(max_pages=1 << 25), dict(max_pages=1 << 24, n_seqs=1000),
               dict(tq=1 << 27), dict(tq=1 << 22, max_pages=1 << 15)):
        assert _call(**kw) == no, kw
    c = B.Cache.__new__(B.Cache)
    for name, v in dict(_k=0x10000, _v=0x10000, _k_scale=0x10000, _v_scale=0x10000, _weight=None, n_pages=9, hkv=4, head_dim=128, page_tokens=64, format=0).items():
        setattr(c, name, v)
    need = B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_SHARED, c, 4, 3, 4, 16)
    assert _call(bytes=need - 1) == full
    assert _call(tq=0, q=None) == B.FCP_OK and _call(n_seqs=0, n_groups=0, groups=None, shared=None) == B.FCP_OK
    for args in ((4, 3, 4, 6), (1 << 20, 1 << 13, 4, 16), (4, 1 << 25, 4, 16), (-1, 3, 4, 16)):
        with pytest.raises(B.FcpError):
            B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_SHARED, c, *args)


# ---- GPU ------------------------------------------------------------------------------------------------------------------------------------
def wide(n_seqs, n_groups, P, D, hkv):
    """Pages of a table with which groups may save 384 MB, so that they are worked together."""
    return (384 << 20) // ((n_seqs - n_groups) * P * hkv * 2 * D) + 1


class Batch:
    """groups: [(common tokens, [(own tokens, new rows), ..]), ..]; the common pages of a group are the first ones of all of its tables.  A sequence's length is common + own.
    narrow: tables of which every sequence is worked by itself."""
    def __init__(self, P, D, hq, hkv, groups, fmt, seed=0, scale=None, narrow=False):
        import torch
        rng = np.random.default_rng(seed + P + D + hq)
        self.kv_len = np.array([c + own for c, seqs in groups for own, _ in seqs], np.int32)
        self.news = [n for _, seqs in groups for _, n in seqs]
        width = max(-(-int(self.kv_len.max()) // P), 1) + 1
        if not narrow:
            width = max(width, wide(len(self.news), len(groups) if len(self.news) > len(groups) else 0, P, D, hkv))
        count = sum(c // P + sum(-(-(c % P + own) // P) for own, _ in seqs) for c, seqs in groups)
        order = list(rng.permutation(count + 2))
        self.pages = np.full((len(self.news), width), -1, np.int32)
        s = 0
        for c, seqs in groups:
            common = [order.pop() for _ in range(c // P)]
            for own, _ in seqs:
                mine = common + [order.pop() for _ in range(-(-(c % P + own) // P))]
                self.pages[s, : len(mine)] = mine
                s += 1
        self.groups = np.cumsum([0] + [len(seqs) for _, seqs in groups]).astype(np.int32)
        self.shared = np.array([c for c, _ in groups], np.int32)
        self.ref = R.RefCache(rng, count + 2, hkv, P, D, fmt)
        for codes in (self.ref.k, self.ref.v):
            codes[:] = R.encode(rng.standard_normal(codes.shape) * (60 if fmt == "e4m3" else 30), fmt)
        self.cu = np.concatenate([[0], np.cumsum(self.news)]).astype(np.int32)
        self.q = R.bf16(rng, self.cu[-1], hq, D)
        self.scale = scale or 1 / np.sqrt(D)
        self.cache = R.to_device(self.ref, torch, B)

    def run(self, groups=None, shared=None, cu=None, fill=float("nan")):
        import torch
        tq, hq, _ = self.q.shape
        groups, shared = self.groups if groups is None else groups, self.shared if shared is None else shared
        n = B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_SHARED, self.cache, len(self.kv_len), self.pages.shape[1], tq, hq)
        scratch = torch.full((n + 65536,), 255, dtype=torch.uint8, device="cuda")
        o, lse = torch.full(self.q.shape, fill, dtype=torch.bfloat16, device="cuda"), torch.full((hq, tq), fill, device="cuda")
        B.fcp_cache_attn_shared(self.cache, dev_bf16(self.q), dev(self.cu if cu is None else cu), dev(self.kv_len), dev(self.pages), dev(groups), dev(shared), self.scale, o, lse,
                                scratch[:n])
        assert (scratch[n:] == 255).all()                    # nothing past scratch of the size that is asked for
        return o.double().cpu().numpy(), lse.double().cpu().numpy()

    def want(self):
        return self.ref.attn(self.q, self.cu, self.kv_len, self.pages, self.scale)

    def check(self, **kw):
        check_attn(self.run(**kw), self.want())


one = lambda *own: [(o, 1) for o in own]
CASES = [  # P, D, hq, hkv, groups
    (16, 64, 4, 4, [(64, one(1, 5))]), (64, 128, 8, 8, [(64, one(1, 1))]), (16, 128, 8, 1, [(300, one(3, 20, 1))]), (32, 64, 32, 8, [(333, one(*range(1, 9)))]),
    (64, 128, 8, 1, [(700, one(2, 70, 130, 1, 9, 64))]), (128, 128, 16, 1, [(515, one(*range(1, 12)))]), (64, 64, 40, 8, [(200, one(1, 2, 3)), (90, one(70, 1)), (450, one(*[7] * 5))]),
    (16, 64, 10, 2, [(50, one(1)), (0, one(4, 5)), (15, one(6, 7)), (16, one(8, 300)), (130, one(1, 1, 1))]), (64, 128, 4, 4, [(2500, one(1, 40))]), (32, 128, 8, 1, [(1900, one(*[5] * 7))]),
    (64, 128, 10, 2, [(150, [(9, 5), (70, 8), (3, 2)])]), (16, 64, 8, 8, [(100, [(40, 40), (33, 20), (65, 65)]), (60, [(20, 7)])]), (64, 128, 40, 8, [(130, [(90, 90), (60, 33)])]),
    (32, 64, 17, 1, [(96, [(3, 3), (0, 0), (10, 0), (4, 1)]), (64, [(5, 0), (7, 0)])]), (128, 64, 8, 2, [(300, [(20, 16), (30, 16)]), (140, [(20, 16), (16, 16)])]),
    (64, 64, 2, 1, [(128, one(*[1] * 70))]), (16, 64, 1, 1, [(33, one(2, 2)) for _ in range(70)])]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P, D, hq, hkv, groups", CASES)
def test_sizes(P, D, hq, hkv, groups, fmt):
    Batch(P, D, hq, hkv, groups, fmt, narrow=True).check()
    b = Batch(P, D, hq, hkv, groups, fmt)
    b.check()
    w = R.check_content(b.cache, b.ref)
    assert np.array_equal(w, b.ref.weight.astype(np.float32))


# more sequences than a block has threads; own parts that are divided, alone and beside short ones; both
MANY_OR_LONG = [
    (16, 64, 2, 2, [(48, one(1, 20)) for _ in range(150)]), (32, 64, 4, 1, [(100, one(*[i % 40 + 1 for i in range(600)])), (0, one(3)), (64, [(5, 0), (9, 1)] * 300)]),
    (16, 64, 16, 1, [(40, [(20, 3), (9, 2), (4, 4)]) for _ in range(100)]), (64, 128, 8, 2, [(200, one(1100, 5, 3000)), (64, one(1025, 1))]), (128, 64, 4, 4, [(1000, one(2500, 1030))]),
    (64, 64, 2, 2, [(64, one(*[1400 if i == 77 else i % 9 + 1 for i in range(300)]))]), (64, 128, 40, 8, [(130, [(1300, 9), (1200, 3)])])]


@pytest.mark.gpu
@pytest.mark.parametrize("P, D, hq, hkv, groups", MANY_OR_LONG)
def test_many_sequences_and_long_ones(P, D, hq, hkv, groups):
    Batch(P, D, hq, hkv, groups, "int8" if P == 64 else "e4m3").check()


@pytest.mark.gpu
def test_many_sequences_whose_tables_fall():
    b = Batch(16, 64, 2, 2, [(48, one(1, 20)) for _ in range(150)], "int8")
    for name, at, to in (("cu", 200, 2 ** 31 - 1), ("cu", 299, 0), ("groups", 100, 301), ("groups", 70, 1), ("groups", 0, -1)):
        table = getattr(b, name).copy()
        table[at] = to
        o, lse = b.run(fill=7.0, **{name: table})
        assert (o == 7).all() and (lse == 7).all(), (name, at)


@pytest.mark.gpu
@pytest.mark.parametrize("count", [1, 3, 5, 200])
@pytest.mark.parametrize("new", [1, 9])
def test_common_pages_are_read_once(count, new):
    """Those of the group's first sequence with rows: what the others' tables say there is not looked at."""
    b = Batch(16, 64, 8, 2, [(48 + 16 * (g % 3), [(5, 0), (new + g % 2, new), (new + 30, new), (new, new)]) for g in range(count)], "int8")
    want = b.want()
    for g in range(count):
        pages = 3 + g % 3
        b.pages[4 * g, :pages] = -1                          # (no rows)
        b.pages[4 * g + 2, :pages], b.pages[4 * g + 3, :pages] = -1, b.pages[(4 * g + 17) % (4 * count), 0]
    check_attn(b.run(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_less_is_shared_than_said(fmt):
    """Lengths that no page ends at, rows that do not see all that is said to be common, negative ones, sequences outside groups, groups of one sequence or of none."""
    b = Batch(32, 64, 8, 2, [(200, [(3, 1), (1, 1), (40, 41), (2, 150)]), (100, one(3, 4, 5)), (64, one(1))], fmt)
    for shared in ([200, 100, 64], [199, 33, 64], [31, 32, 0], [-5, 1000, 7], [2 ** 31 - 1, 96, -2 ** 31]):
        b.check(shared=np.array(shared))                     # (no row sees tokens past the pages that are really common before its own)
    b.check(groups=[4, 7], shared=[96])
    b.check(groups=[0, 0, 4, 4, 7], shared=[9, 192, 9, 96])
    b.check(groups=[1, 3, 3], shared=[192, 100])
    b.check(groups=[0], shared=[])
    b.check(groups=[8], shared=[])


@pytest.mark.gpu
def test_rows_do_not_see_past_themselves():
    """Said to be common: more than a sequence has before its new rows.  What they share then are the tokens before."""
    b = Batch(16, 64, 4, 2, [(160, [(0, 100), (30, 1), (0, 170)])], "int8")
    b.check()
    b = Batch(16, 64, 4, 2, [(160, [(0, 100), (30, 1)])], "int8")
    b.check()


@pytest.mark.gpu
def test_empty_sequences():
    b = Batch(16, 64, 4, 2, [(0, one(0, 5)), (48, one(1, 9))], "int8")
    b.check()
    got = b.run()
    assert (got[0][0] == 0).all() and np.isneginf(got[1][:, 0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("groups", [[(200, one(3, 40, 2))], [(200, one(*range(1, 30)))], [(200, [(40, 30), (50, 35)])]])
@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_that_are_not_there(fmt, groups):
    """In the common part and in a sequence's own: seen by nobody."""
    b = Batch(32, 64, 4, 2, groups, fmt)
    b.pages[:, 1], b.pages[:, 4] = -1, 10 ** 6
    b.pages[1, 6] = -7
    b.check()
    b.pages[:] = -1
    b.check()


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("groups", [[(200, one(3, 40, 2)), (150, one(9, 1))], [(1500, one(*range(1, 30))), (64, one(1, 1))], [(200, [(40, 30), (50, 35)]), (64, [(20, 20), (9, 9)])]])
def test_nan_reaches_only_the_rows_that_see_it(D, groups):
    import torch
    b = Batch(64, D, 4, 2, groups, "e4m3")
    end, own = len(groups[0][1]), groups[0][0] // 64         # sequences of the first group; the first page of a sequence's own
    b.ref.v[b.pages[0, 1], 0, 5, 3] = 127                    # a common value: every row of the group, that channel
    last = int(b.kv_len[1]) - 1
    b.ref.v[b.pages[1, last // 64], 1, last % 64, 17] = 255  # a sequence's last value: its last row
    b.ref.v[b.pages[1, last // 64], :, last % 64 + 1:] = 127
    b.ref.k[b.pages[2 if end > 2 else 0, own], 0, 0, 9] = 127     # a sequence's own key
    b.cache = R.to_device(b.ref, torch, B)
    got, want = b.run(), b.want()
    assert np.isnan(want[0][: b.cu[end]]).any() and not np.isnan(want[0][b.cu[end]:]).any()
    check_attn(got, want)


@pytest.mark.gpu
def test_scores_that_differ_widely():
    """The greatest score in the common part, in the own part; e^-80 beside 1."""
    for seed in range(3):
        Batch(64, 64, 4, 4, [(640, one(1, 64, 200, 9))], "e4m3", seed=seed, scale=2.0).check()


@pytest.mark.gpu
def test_rows_outside_sequences_and_tables_that_fall():
    """Rows before the first and behind the last sequence stay; where cu_seqlens or groups fall, or groups name sequences that are not there, nothing is written."""
    b = Batch(32, 64, 4, 2, [(96, one(5, 6, 7)), (64, one(1, 2))], "int8")
    whole = b.run()
    b.q = np.concatenate([b.q[:2] * 0 + 1, b.q, b.q[:3]])
    o, lse = b.run(cu=b.cu + 2, fill=7.0)
    assert np.array_equal(o[2:7], whole[0]) and np.array_equal(lse[:, 2:7], whole[1])
    assert (o[:2] == 7).all() and (o[7:] == 7).all() and (lse[:, :2] == 7).all() and (lse[:, 7:] == 7).all()
    for kw in (dict(cu=[0, 2, 1, 3, 4, 5]), dict(cu=[0, 2147483647, -2147483648, 3, 4, 5]), dict(groups=[0, 3, 2]), dict(groups=[-1, 3, 5]), dict(groups=[0, 3, 6]), dict(groups=[3, 0, 5])):
        o, lse = b.run(fill=7.0, **kw)
        assert (o == 7).all() and (lse == 7).all(), kw


@pytest.mark.gpu
@pytest.mark.parametrize("news, seqs", [(1, 4), (1, 40), (20, 5)])
def test_repeats_and_follows_its_tables_in_graphs(news, seqs):
    """Two graphs with scratch of their own beside eager calls on another stream; lengths, groups and queries change between replays."""
    import torch
    b = Batch(64, 128, 16, 4, [(500, [(40 + i, news) for i in range(seqs)]), (130, [(30, news)] * 3)], "e4m3")
    n = B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_SHARED, b.cache, len(b.kv_len), b.pages.shape[1], len(b.q), 16)
    space = lambda: torch.empty(n, dtype=torch.uint8, device="cuda")
    q, cu, lens, pages, groups, shared = dev_bf16(b.q), dev(b.cu), dev(b.kv_len), dev(b.pages), dev(b.groups), dev(b.shared)
    outs = [(torch.empty_like(q), torch.empty(16, len(b.q), device="cuda"), space()) for _ in range(3)]
    call = lambda o: B.fcp_cache_attn_shared(b.cache, q, cu, lens, pages, groups, shared, b.scale, *o)
    call(outs[0])
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, o in zip(graphs, outs[1:]):
        with torch.cuda.graph(g):
            call(o)
    side = torch.cuda.Stream()
    for i in range(4):
        lens.sub_(1)
        q.mul_(0.9)
        if i == 2:
            shared.copy_(dev([448, 0]))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(outs[0])
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[0][j], o[j]) for o in outs[1:] for j in range(2)), i
    ordinary = torch.empty_like(q), torch.empty(16, len(b.q), device="cuda")
    w = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_ATTN, b.cache, len(b.kv_len), b.pages.shape[1], len(b.q), 16), dtype=torch.uint8, device="cuda")
    B.fcp_cache_attn(b.cache, q, cu, lens, pages, b.scale, *ordinary, w)
    # both are off by a bf16 rounding of O and, with many rows, of each probability: at most 2^-8 of the greatest |v| in a row each
    assert float((ordinary[0].float() - outs[0][0].float()).abs().max()) <= 2.0 ** -6 * 8 and float((ordinary[1] - outs[0][1]).abs().max()) < 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("fmt, least", [("e4m3", -100), ("e4m3", 0), ("int8", -100)])        # (codes from -100 on: -1 is NaN in e4m3, and nearly every row sees one)
def test_pages_past_the_32nd_bit(fmt, least):
    """The last pages of a pool whose keys take more than 2^32 bytes: bit for bit what the same pages give in a small pool."""
    import torch
    P, D, hkv, hq, used = 128, 128, 8, 8, 16
    n_big = (1 << 32) // (P * D * hkv) + used
    view = lambda t: t.view(torch.float8_e4m3fn) if fmt == "e4m3" else t
    g = torch.Generator(device="cuda").manual_seed(3)
    small = [torch.randint(least, 100, s, generator=g, device="cuda").to(torch.int8) for s in ((used, hkv, P, D), (used, hkv, P // 16, D, 16))]
    q = torch.randn(41, hq, D, generator=g, device="cuda").to(torch.bfloat16)
    results = []
    for n in (used, n_big):
        k, v = (torch.empty(n, *x.shape[1:], dtype=torch.int8, device="cuda") for x in small)
        for to, x in ((k, small[0]), (v, small[1])):
            to[n - used:] = x
        ones = torch.ones(n, hkv, device="cuda") / 64
        cache = B.Cache(view(k), view(v), ones, ones)
        pages = torch.full((3, wide(3, 1, P, D, hkv)), -1, dtype=torch.int32, device="cuda")
        pages[:, :5] = dev(np.array([[5, 0, 3, 7, -1], [5, 0, 3, 1, 9], [2, 8, -1, -1, -1]], np.int32)) + (n - used)
        for cu in ([0, 1, 2, 3], [0, 20, 40, 41]):
            m = cu[-1]
            o, lse = torch.empty(m, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(hq, m, device="cuda")
            w = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_SHARED, cache, *pages.shape, m, hq), dtype=torch.uint8, device="cuda")
            B.fcp_cache_attn_shared(cache, q[:m].contiguous(), dev(cu), dev([500, 600, 200]), pages, dev([0, 2]), dev([384]), 0.05, o, lse, w)
            results.append((o, lse))
        del cache, k, v
    for a, b in zip(results[:2], results[2:]):
        assert torch.equal(a[0].view(torch.int16), b[0].view(torch.int16)) and torch.equal(a[1].view(torch.int32), b[1].view(torch.int32))
        assert torch.isfinite(a[1]).all() == (fmt == "int8" or least == 0)


@pytest.mark.gpu
def test_small_tables_are_worked_by_themselves():
    """Whatever groups and shared_len hold: bit for bit what fcp_cache_attn gives."""
    import torch
    b = Batch(32, 64, 8, 2, [(192, one(3, 4, 5)), (64, one(1, 2))], "e4m3", narrow=True)
    q, cu, lens, pages = dev_bf16(b.q), dev(b.cu), dev(b.kv_len), dev(b.pages)
    o, lse = torch.empty_like(q), torch.empty(8, len(b.q), device="cuda")
    w = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_ATTN, b.cache, len(b.kv_len), b.pages.shape[1], len(b.q), 8), dtype=torch.uint8, device="cuda")
    B.fcp_cache_attn(b.cache, q, cu, lens, pages, b.scale, o, lse, w)
    for kw in (dict(), dict(groups=[0, 4, 2]), dict(groups=[-5, 9, 9]), dict(shared=[10 ** 6, -3]), dict(groups=[0], shared=[])):
        got = b.run(**kw)
        assert np.array_equal(got[0], o.double().cpu().numpy()) and np.array_equal(got[1], lse.double().cpu().numpy())


@pytest.mark.gpu
def test_queries_that_are_slices_of_wider_rows():
    import torch
    b = Batch(32, 64, 6, 2, [(96, one(5, 6, 7))], "int8")
    wide = torch.full((3, 6 * 64 + 200), float("nan"), dtype=torch.bfloat16, device="cuda")
    sliced = wide[:, 8: 8 + 384].unflatten(1, (6, 64))
    sliced.copy_(dev_bf16(b.q))
    out = []
    for x in (dev_bf16(b.q), sliced):
        o, lse = torch.empty(3, 6, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(6, 3, device="cuda")
        w = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_SHARED, b.cache, 3, b.pages.shape[1], 3, 6), dtype=torch.uint8, device="cuda")
        B.fcp_cache_attn_shared(b.cache, x, dev(b.cu), dev(b.kv_len), dev(b.pages), dev(b.groups), dev(b.shared), b.scale, o, lse, w)
        out.append((o, lse))
    assert all(torch.equal(x, y) for x, y in zip(*out))
    with pytest.raises(ValueError):
        B.fcp_cache_attn_shared(b.cache, x, dev(b.cu), dev(b.kv_len), dev(b.pages), dev([0]), dev(b.shared), b.scale, o, lse, w)
    with pytest.raises(ValueError):
        B.fcp_cache_attn_shared(b.cache, x, dev(b.cu), dev(b.kv_len), dev(b.pages), dev(b.groups), dev(b.shared).long(), b.scale, o, lse, w)
