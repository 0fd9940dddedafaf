"""The paged 8-bit cache: appending, attention, weights and eviction against plain forms in 64 bits (tests/cache_ref.py), and the refusals (on the CPU)."""
import ctypes

import numpy as np
import pytest

import cache_ref as R
from paper_2602_21788_amd import binding as B

FORMATS = ["e4m3", "int8"]


# ---- CPU ------------------------------------------------------------------------------------------------------------------------------------
def test_reference_codes():
    """The oracle's own rounding: every value is its own code, midpoints go to even codes, the ends saturate."""
    for fmt in FORMATS:
        codes = np.arange(256, dtype=np.uint8)
        v = R.decode(codes, fmt)
        fine = ~np.isnan(v) & (codes != 128)
        assert np.array_equal(R.decode(R.encode(v[fine], fmt), fmt), v[fine])
        up = np.unique(v[fine & (v >= 0)])
        mid = (up[1:] + up[:-1]) / 2
        c = R.encode(mid, fmt)
        assert (c % 2 == 0).all()
        assert R.decode(R.encode(np.array([1e9, -np.inf]), fmt), fmt).tolist() == [R.MOST[fmt], -R.MOST[fmt]]
    assert R.exponent(np.array([448.0]), "e4m3") == 0 and R.exponent(np.array([448.1]), "e4m3") == 1
    assert R.exponent(np.array([127.0, np.nan, np.inf]), "int8") == 0 and R.exponent(np.array([127.5]), "int8") == 1
    assert R.exponent(np.zeros(3), "int8") == R.LEAST == R.exponent(np.array([1e-40]), "e4m3")


def test_reference_rows_and_order():
    rng = np.random.default_rng(0)
    x = rng.integers(0, 256, (3, 2, 32, 64), dtype=np.uint8)
    v = R.v_order(x)
    assert v.shape == (3, 2, 2, 64, 16) and v[1, 0, 1, 7, 5] == x[1, 0, 21, 7] and np.array_equal(R.v_back(v), x)


class Call:
    """Calls with addresses that nobody looks at: every one below fails first, or has nothing to do."""
    fake = 0x10000

    def __init__(self, **kw):
        f = self.fake
        self.c = B.Cache.__new__(B.Cache)
        for name, v in dict(_k=f, _v=f, _k_scale=f, _v_scale=f, _weight=f, n_pages=9, hkv=4, head_dim=128, page_tokens=64, format=0).items():
            setattr(self.c, name, kw.pop(name, v))
        self.kw = kw

    def arg(self, name, v):
        return self.kw.get(name, v)

    def ref(self):
        return None if self.kw.get("no_cache") else ctypes.byref(self.c)

    def append(self):
        a, f = self.arg, self.fake
        return B.lib().fcp_cache_append(self.ref(), a("k", f), a("k_row", 512), a("v", f), a("v_row", 512), a("n_rows", 5), a("cu", f), a("kv_len", f),
                                        a("pages", f), a("n_seqs", 2), a("max_pages", 3), None)

    def attn(self):
        a, f = self.arg, self.fake
        return B.lib().fcp_cache_attn(self.ref(), a("q", f), a("q_row", 2048), a("tq", 2), a("hq", 16), a("cu", f), a("kv_len", f), a("pages", f), a("n_seqs", 2),
                                      a("max_pages", 3), a("scale", 0.1), a("weigh", 0), a("o", f), a("lse", f), a("scratch", f), a("bytes", 1 << 40), None)

    def weigh(self):
        a, f = self.arg, self.fake
        return B.lib().fcp_cache_weigh(self.ref(), a("q", f), a("q_row", 2048), a("tq", 2), a("hq", 16), a("lse", f), a("cu", f), a("kv_len", f), a("pages", f),
                                       a("n_seqs", 2), a("max_pages", 3), a("scale", 0.1), None)

    def evict(self):
        a, f = self.arg, self.fake
        return B.lib().fcp_cache_evict(self.ref(), a("pages", f), a("kv_len", f), a("n_seqs", 2), a("max_pages", 3), a("new_pages", f), a("max_new", 2), a("budget", 128),
                                       a("first", 4), a("recent", 32), a("kept", f), a("new_len", f + 64), a("scratch", f), a("bytes", 1 << 40), None)


def test_refusals_come_before_any_device_work():
    bad, no, full = B.FCP_ERR_INVALID_ARG, B.FCP_ERR_UNSUPPORTED, B.FCP_ERR_CAPACITY
    for op in ("append", "attn", "weigh", "evict"):
        call = lambda **kw: getattr(Call(**kw), op)()
        assert call(no_cache=True) == bad
        assert call(_k=None) == bad and call(_v_scale=None) == bad and call(n_pages=0) == bad and call(hkv=0) == bad
        assert call(_k=0x10008) == bad and b"aligned" in B.lib().fcp_last_error()
        assert call(head_dim=96) == no and call(page_tokens=48) == no and call(page_tokens=8) == no and call(page_tokens=256) == no
        assert call(format=2) == no and call(hkv=5000) == no
        assert call(n_seqs=-1) == bad and call(max_pages=-1) == bad and call(kv_len=None) == bad and call(pages=None) == bad
        assert call(n_seqs=(1 << 20) + 1) == no
        assert call(n_seqs=0) == 0
    assert Call(n_rows=-1).append() == bad and Call(k=None).append() == bad and Call(cu=None).append() == bad
    assert Call(k_row=511).append() == bad and Call(v_row=516).append() == bad and Call(v=Call.fake + 2).append() == bad
    assert Call(n_rows=0, k=None).append() == 0 and Call(max_pages=0, pages=None).append() == 0
    for op in ("attn", "weigh"):
        call = lambda **kw: getattr(Call(**kw), op)()
        assert call(hq=6) == no and call(hq=0) == no and call(tq=-1) == bad and call(cu=None) == bad and call(q=None) == bad
        assert call(q_row=2047) == bad and call(q_row=2052) == bad and call(scale=0.0) == bad and call(scale=float("nan")) == bad
        assert call(lse=None) == bad and call(tq=0, q=None) == 0
        assert call(tq=1 << 30) == no
    assert Call(o=None).attn() == bad and Call(weigh=2).attn() == bad and Call(weigh=1, _weight=None).attn() == bad
    assert Call(scratch=None).attn() == bad and Call(scratch=Call.fake + 16).attn() == bad and Call(bytes=100).attn() == full
    assert Call(_weight=None).weigh() == bad and Call(_weight=None).evict() == bad
    assert Call(budget=0, first=0, recent=0).evict() == bad and Call(first=97).evict() == bad and Call(first=-1).evict() == bad
    assert Call(new_pages=None).evict() == bad and Call(kept=None).evict() == bad and Call(new_len=Call.fake).evict() == bad
    assert Call(max_new=1).evict() == full and Call(scratch=Call.fake + 1).evict() == bad and Call(bytes=1).evict() == full


def test_tables_are_bounded():
    """A token's place is a 32-bit number, and tiles past the last one are looked at."""
    for op in ("append", "attn", "weigh", "evict"):
        for page, pages in ((128, (1 << 23) + 1), (16, (1 << 26) + 1), (16, 1 << 30)):
            assert getattr(Call(page_tokens=page, max_pages=pages), op)() == B.FCP_ERR_UNSUPPORTED and b"2^30 tokens" in B.lib().fcp_last_error()


def test_scratch_sizes():
    c = Call().c
    for which in (B.FCP_SCRATCH_CACHE_ATTN, B.FCP_SCRATCH_CACHE_WEIGH, B.FCP_SCRATCH_CACHE_EVICT):
        n = B.fcp_cache_scratch_bytes(which, c, 4, 100, 4, 16)
        assert n >= 256 and n % 256 == 0
        with pytest.raises(B.FcpError):
            B.fcp_cache_scratch_bytes(which, c, -1, 100, 4, 16)
    with pytest.raises(B.FcpError):
        B.fcp_cache_scratch_bytes(0, c, 4, 100, 4, 16)
    with pytest.raises(B.FcpError):
        B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_ATTN, c, 4, 100, 4, 6)


# ---- GPU ------------------------------------------------------------------------------------------------------------------------------------
def dev(a, dt=np.int32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dt)).cuda()


def dev_bf16(a):
    import torch
    return torch.from_numpy(a.astype(np.float32)).cuda().to(torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P,D,hkv,kv_len,news", [
    (16, 64, 2, [1], [1]), (64, 128, 1, [64, 65, 1], [1, 1, 1]), (16, 128, 3, [40, 7, 33, 16], [3, 0, 33, 1]), (128, 64, 2, [300, 5], [129, 5]),
    (32, 128, 2, [31, 100, 64], [31, 70, 17]), (64, 64, 5, [200] * 3, [1, 2, 130]), (16, 128, 1, [19], [25])])
def test_append(P, D, hkv, kv_len, news, fmt):
    import torch
    rng = np.random.default_rng(P + D + len(kv_len))
    pages, total = R.tables(rng, kv_len, P, extra=1)
    ref = R.RefCache(rng, total, hkv, P, D, fmt)
    cache = R.to_device(ref, torch, B)
    cu = np.concatenate([[0], np.cumsum(news)])
    # magnitudes around those that are cached, so that some pages grow and others do not
    k, v = (R.bf16(rng, cu[-1], hkv, D, scale=1.0) * np.exp2(rng.integers(-6, 6, (cu[-1], hkv, 1))) for _ in range(2))
    B.fcp_cache_append(cache, dev_bf16(k), dev_bf16(v), dev(cu), dev(kv_len), dev(pages))
    ref.append(k, v, cu, kv_len, pages)
    assert np.array_equal(R.check_content(cache, ref), ref.weight.astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_append_of_strided_rows_and_of_values_that_are_not_finite(fmt):
    import torch
    rng = np.random.default_rng(5)
    P, D, hkv, kv_len, news = 32, 64, 2, [70, 20, 64], [40, 20, 1]
    pages, total = R.tables(rng, kv_len, P)
    ref = R.RefCache(rng, total, hkv, P, D, fmt)
    cache = R.to_device(ref, torch, B)
    cu = np.concatenate([[0], np.cumsum(news)])
    k, v = R.bf16(rng, cu[-1], hkv, D), R.bf16(rng, cu[-1], hkv, D)
    k[3, 0, 5], k[4, 1, 6], v[50, 1, 63], v[7, 0, 0] = np.inf, np.nan, -np.inf, np.nan
    k[60], v[59] = 0.0, 1e-39                        # a page's only row all zeros; magnitudes below the least scale
    v[60], v[59, 0, 0] = 3.3e38, np.nan
    k, v = (torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).float().numpy().astype(np.float64) for x in (k, v))
    both = torch.full((cu[-1], 2 * hkv * D + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    kd, vd = both[:, : hkv * D].unflatten(1, (hkv, D)), both[:, hkv * D: 2 * hkv * D].unflatten(1, (hkv, D))
    kd.copy_(dev_bf16(k)), vd.copy_(dev_bf16(v))
    B.fcp_cache_append(cache, kd, vd, dev(cu), dev(kv_len), dev(pages))
    ref.append(k, v, cu, kv_len, pages)
    R.check_content(cache, ref)


@pytest.mark.gpu
def test_append_writes_no_page_that_is_not_there():
    """Numbers outside the pool, sequences that begin past their table, offsets past the rows: skipped."""
    import torch
    rng = np.random.default_rng(6)
    P, D, hkv = 16, 64, 1
    ref = R.RefCache(rng, 6, hkv, P, D, "int8")
    cache = R.to_device(ref, torch, B)
    pages = np.array([[0, -1, 2], [7, 1000000, 3], [4, 5, -2147483648]], np.int32)
    kv_len, cu = [48, 40, 33], np.array([0, 48, 58, 60])
    k, v = R.bf16(rng, 60, hkv, D), R.bf16(rng, 60, hkv, D)
    B.fcp_cache_append(cache, dev_bf16(k), dev_bf16(v), dev(cu), dev(kv_len), dev(pages))
    ref.append(k, v, cu, kv_len, pages)
    R.check_content(cache, ref)
    # tables with nonsense in them: nothing is read or written outside; here nothing may change
    for lens, cus in (([0, 0, 0], [0, 1, 2, 3]), ([-5, 0, -2147483648], [0, 20, 40, 60]), ([16, 16, 16], [60, 2000000000, 61, -4])):
        B.fcp_cache_append(cache, dev_bf16(k), dev_bf16(v), dev(cus), dev(lens), dev(pages))
        R.check_content(cache, ref)


ATTN = [  # P, D, hq, hkv, kv_len, news
    (16, 64, 4, 4, [1], [1]), (64, 128, 8, 1, [64, 65, 1], [1, 1, 1]), (16, 128, 6, 2, [40, 7, 0, 16, 300], [1, 1, 1, 1, 1]),
    (128, 64, 32, 8, [777], [1]), (32, 128, 10, 2, [31, 260], [3, 2]), (64, 128, 40, 8, [200, 90], [90, 90]), (64, 64, 8, 8, [130], [130]),
    (16, 64, 17, 1, [513, 20], [5, 0]), (32, 128, 4, 4, [3, 2], [5, 2]), (64, 128, 32, 8, [2500, 3], [1, 1]), (16, 128, 24, 1, [77], [33])]


def attn_case(P, D, hq, hkv, kv_len, news, fmt, seed=0, scale=None):
    import torch
    rng = np.random.default_rng(seed + P + D + hq)
    pages, total = R.tables(rng, kv_len, P, extra=1)
    ref = R.RefCache(rng, total, hkv, P, D, fmt)
    for codes in (ref.k, ref.v):                    # bell-shaped codes: random ones nearly all lie at the upper end of e4m3's range
        codes[:] = R.encode(rng.standard_normal(codes.shape) * (60 if fmt == "e4m3" else 30), fmt)
    cu = np.concatenate([[0], np.cumsum(news)])
    q = R.bf16(rng, cu[-1], hq, D)
    return ref, R.to_device(ref, torch, B), pages, cu, q, scale or 1 / np.sqrt(D)


def run_attn(cache, q, cu, kv_len, pages, scale, weigh):
    import torch
    which = B.FCP_SCRATCH_CACHE_WEIGH if weigh else B.FCP_SCRATCH_CACHE_ATTN
    scratch = torch.full((B.fcp_cache_scratch_bytes(which, cache, len(kv_len), pages.shape[1], q.shape[0], q.shape[1]),), 255, dtype=torch.uint8, device="cuda")
    o = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((q.shape[1], q.shape[0]), float("nan"), device="cuda")
    B.fcp_cache_attn(cache, dev_bf16(q), dev(cu), dev(kv_len), dev(pages), scale, o, lse, scratch, weigh=weigh)
    return o.double().cpu().numpy(), lse.double().cpu().numpy()


def check_attn(got, want):
    """A score is off by at most `units` 2^-24 (its product) and 4 * 2^-24 of itself (scaling, exponential's argument); the probabilities by twice that, and by half a
    step of bf16 for the product; O by half a step more."""
    (o, lse), (O, LSE, _, absv, units) = got, want
    assert np.array_equal(np.isnan(o), np.isnan(O)) and np.array_equal(np.isnan(lse), np.isnan(LSE))
    empty = np.isneginf(LSE)
    assert np.array_equal(np.isneginf(lse), empty) and (o.transpose(1, 0, 2)[empty] == 0).all()
    eps = (units + 8 * np.abs(np.where(empty, 0, LSE)) + 16) * 2.0 ** -24
    fine = ~empty & ~np.isnan(LSE)
    assert (np.abs(lse[fine] - LSE[fine]) <= eps[fine]).all()
    tol = absv * (2.0 ** -8 + 2 * eps.T[..., None]) + np.abs(O) * 2.0 ** -8 + 1e-30
    ok = np.isnan(O) | (np.abs(o - O) <= tol)
    assert ok.all(), float(np.nanmax(np.abs(o - O) / tol))
    return eps


def check_weight(got, before, want, eps, rows):
    """Sums of `rows` probabilities, each off by 2 eps of itself, and the sum's own roundings."""
    assert (np.abs(got - (before + want)) <= want * (2 * eps[np.isfinite(eps)].max() + 1e-6) + (before + want) * (rows + 2) * 2.0 ** -24 + 1e-30).all()


@pytest.mark.gpu
@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news", ATTN)
def test_attention_over_the_cache(P, D, hq, hkv, kv_len, news, fmt, weigh):
    ref, cache, pages, cu, q, scale = attn_case(P, D, hq, hkv, kv_len, news, fmt)
    got = run_attn(cache, q, cu, kv_len, pages, scale, weigh)
    want = ref.attn(q, cu, kv_len, pages, scale)
    eps = check_attn(got, want)
    w = R.check_content(cache, ref)
    if weigh:
        check_weight(w, ref.weight, want[2], eps, max(news) * hq // hkv)
    else:
        assert np.array_equal(w, ref.weight.astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news", ATTN)
def test_weights_of_known_sums(P, D, hq, hkv, kv_len, news, fmt):
    import torch
    ref, cache, pages, cu, q, scale = attn_case(P, D, hq, hkv, kv_len, news, fmt, seed=1)
    _, LSE, want, _, units = ref.attn(q, cu, kv_len, pages, scale)
    lse = LSE.astype(np.float32)
    B.fcp_cache_weigh(cache, dev_bf16(q), torch.from_numpy(lse).cuda(), dev(cu), dev(kv_len), dev(pages), scale)
    # (the sums as floats: their own rounding is part of the input)
    _, _, want, _, _ = ref.attn(q, cu, kv_len, pages, scale, lse_in=lse.astype(np.float64))
    eps = (units + 8 * np.abs(np.where(np.isneginf(LSE), 0, LSE)) + 16) * 2.0 ** -24
    check_weight(R.check_content(cache, ref), ref.weight, want, eps, max(news) * hq // hkv)


@pytest.mark.gpu
@pytest.mark.parametrize("news", [[1, 1], [3, 2], [60, 40]])
@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_past_missing_pages(fmt, news):
    """Pages that are not there are seen by nobody; a sequence of nothing else gets O = 0, LSE = -inf."""
    kv_len = [150, 70]
    ref, cache, pages, cu, q, scale = attn_case(32, 64, 4, 2, kv_len, news, fmt)
    pages[0, 1], pages[0, 4], pages[1, :] = -1, 10 ** 6, -7
    got = run_attn(cache, q, cu, kv_len, pages, scale, True)
    want = ref.attn(q, cu, kv_len, pages, scale)
    assert np.isneginf(want[1][:, cu[1]:]).all()
    check_weight(R.check_content(cache, ref), ref.weight, want[2], check_attn(got, want), max(news) * 2)


@pytest.mark.gpu
@pytest.mark.parametrize("news", [[1], [4], [70]])
@pytest.mark.parametrize("bad_key", [False, True])
def test_nan_in_the_cache_reaches_only_the_rows_that_see_it(news, bad_key):
    """NaN codes past the last token, in a page's unused slots, and in a key or value that only the last rows see."""
    import torch
    kv_len = [90]
    ref, cache, pages, cu, q, scale = attn_case(64, 128, 4, 2, kv_len, news, "e4m3")
    for codes in (ref.k, ref.v):
        codes[pages[0, 1], :, 26:] = 127
    (ref.k if bad_key else ref.v)[pages[0, 1], 1, 25, 11] = 255      # the last token, KV head 1
    cache = R.to_device(ref, torch, B)
    got = run_attn(cache, q, cu, kv_len, pages, scale, False)
    want = ref.attn(q, cu, kv_len, pages, scale)
    assert np.isnan(want[0]).any() and not np.isnan(want[0][:-1]).any() and not np.isnan(want[0][:, :2]).any()
    check_attn(got, want)


@pytest.mark.gpu
def test_nan_among_many_items():
    """More (sequence, KV head, block of rows) than blocks run at once, so blocks work several in turn: what one saw does not reach the next.  Some sequences are shorter than
    their new rows, so that whole blocks of rows see nothing."""
    import torch
    kv_len = [8 if i % 9 == 4 else 80 + 13 * i % 110 for i in range(60)]
    news = [90 if i % 9 == 4 else 70 for i in range(60)]
    ref, cache, pages, cu, q, scale = attn_case(32, 64, 10, 5, kv_len, news, "e4m3")
    for i in range(0, 60, 2):
        t, head, channel = kv_len[i] - 1 - i % 3, i % 5, 7 * i % 64
        ref.v[pages[i, t // 32], head, t % 32, channel] = 127
    cache = R.to_device(ref, torch, B)
    got = run_attn(cache, q, cu, kv_len, pages, scale, False)
    want = ref.attn(q, cu, kv_len, pages, scale)
    assert 60 < np.isnan(want[0]).sum() < 400 and np.isneginf(want[1]).any()
    check_attn(got, want)


@pytest.mark.gpu
def test_scores_that_differ_widely():
    """The running maximum rises many times and falls behind by far: e^-80 beside 1."""
    ref, cache, pages, cu, q, scale = attn_case(64, 64, 4, 4, [1000, 640], [1, 1], "e4m3", scale=2.0)
    check_attn(run_attn(cache, q, cu, [1000, 640], pages, scale, False), ref.attn(q, cu, [1000, 640], pages, scale))


@pytest.mark.gpu
@pytest.mark.parametrize("news", [1, 20])
def test_attention_repeats_and_follows_its_tables_in_a_graph(news):
    import torch
    kv_len = [500, 33, 129, 1024]
    ref, cache, pages, cu, q, scale = attn_case(64, 128, 16, 4, kv_len, [news] * 4, "int8")
    n = B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_WEIGH, cache, 4, pages.shape[1], q.shape[0], 16)
    scratch = torch.empty(n, dtype=torch.uint8, device="cuda")
    qd, cud, lend, pd = dev_bf16(q), dev(cu), dev(kv_len), dev(pages)
    outs = [(torch.empty_like(qd), torch.empty(16, q.shape[0], device="cuda")) for _ in range(2)]
    call = lambda o: B.fcp_cache_attn(cache, qd, cud, lend, pd, scale, o[0], o[1], scratch, weigh=True)
    call(outs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[1])
    side = torch.cuda.Stream()
    for i in range(4):
        lend.sub_(torch.tensor([7, 1, 64, 100], dtype=torch.int32, device="cuda"))
        qd.mul_(0.9)
        cache.weight.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(outs[0])
        torch.cuda.current_stream().wait_stream(side)
        first = cache.weight.clone()
        cache.weight.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and torch.equal(first, cache.weight), i


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P,D,hkv,kv_len,budget,first,recent", [
    (16, 64, 2, [1], 1, 0, 0), (16, 64, 2, [100, 40, 0, 41], 40, 2, 8), (64, 128, 1, [700], 65, 0, 1), (32, 128, 3, [333, 64, 90], 64, 4, 60),
    (128, 64, 2, [1000, 129], 300, 8, 100), (64, 64, 1, [5000], 1111, 4, 200), (16, 128, 2, [77, 77], 77, 0, 77), (16, 64, 1, [60], 17, 0, 0),
    (32, 64, 2, [40000, 30, 16389, 9001], 9000, 5, 100), (128, 64, 1, [33000], 32000, 0, 0), (16, 64, 1, [70001, 69000], 20, 4, 16)])
def test_evict(P, D, hkv, kv_len, budget, first, recent, fmt):
    import torch
    rng = np.random.default_rng(budget)
    pages, n_old = R.tables(rng, kv_len, P)
    new_counts = [-(-min(n, budget) // P) for n in kv_len]
    new_pages = np.full((len(kv_len), max(-(-min(budget, pages.shape[1] * P) // P), 1) + 1), -1, np.int32)
    order, at = n_old + rng.permutation(sum(new_counts) + 1), 0
    for s, c in enumerate(new_counts):
        new_pages[s, :c] = order[at: at + c]
        at += c
    ref = R.RefCache(rng, n_old + sum(new_counts) + 1, hkv, P, D, fmt)
    if len(kv_len) > 1 and kv_len[0] > 60:            # orders that are easily taken wrongly
        ref.weight[pages[0, 1], 0, 3: 9] = [np.nan, np.inf, 0.0, -0.0, -1.0, 1e-42]
        if fmt == "e4m3":
            ref.k[pages[0, 0], 0, 1, 2] = 127
    cache = R.to_device(ref, torch, B)
    kept = torch.full((len(kv_len), hkv, budget), 12345, dtype=torch.int32, device="cuda")
    new_len = torch.full((len(kv_len),), 12345, dtype=torch.int32, device="cuda")
    scratch = torch.full((B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_EVICT, cache, len(kv_len), pages.shape[1]),), 255, dtype=torch.uint8, device="cuda")
    for again in range(2):                            # (the old pages still hold everything)
        B.fcp_cache_evict(cache, dev(pages), dev(kv_len), dev(new_pages), budget, first, recent, kept, new_len, scratch)
    want_kept, want_len = ref.evict(pages, kv_len, new_pages, budget, first, recent)
    assert np.array_equal(new_len.cpu().numpy(), want_len)
    assert np.array_equal(kept.cpu().numpy(), want_kept)
    w = R.check_content(cache, ref)
    assert np.array_equal(w, ref.weight.astype(np.float32), equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [5000, 30000])
@pytest.mark.parametrize("kind", ["equal", "two", "near"])
def test_evict_of_weights_that_share_their_upper_bits(n, kind):
    """One value, two values, and values whose upper bits are all alike: the kept are the greatest, and of equal ones the lowest."""
    import torch
    P, D, budget, first, recent = 64, 64, n // 3, 3, 50
    counts, new = -(-n // P), -(-budget // P)
    rng = np.random.default_rng(n)
    w = {"equal": np.zeros(n), "two": rng.integers(0, 2, n) * 0.5, "near": 1 + rng.integers(0, 3000, n) * 2.0 ** -23}[kind].astype(np.float32)
    weight = np.zeros((counts + new, 1, P), np.float32)
    weight.reshape(-1)[:n] = w
    z = lambda *s, dt=torch.int8: torch.zeros(*s, dtype=dt, device="cuda")
    cache = B.Cache(z(counts + new, 1, P, D), z(counts + new, 1, P // 16, D, 16), z(counts + new, 1, dt=torch.float32) + 1, z(counts + new, 1, dt=torch.float32) + 1,
                    torch.from_numpy(weight).cuda())
    pages, new_pages = dev(np.arange(counts)[None]), dev(np.arange(counts, counts + new)[None])
    kept, new_len = z(1, 1, budget, dt=torch.int32), z(1, dt=torch.int32)
    scratch = torch.full((B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_EVICT, cache, 1, counts),), 255, dtype=torch.uint8, device="cuda")
    B.fcp_cache_evict(cache, pages, dev([n]), new_pages, budget, first, recent, kept, new_len, scratch)
    order = np.argsort(-w[first: n - recent], kind="stable")[: budget - first - recent] + first
    assert np.array_equal(kept.cpu().numpy()[0, 0], np.sort(np.concatenate([np.arange(first), order, np.arange(n - recent, n)])))
    assert np.array_equal(cache.weight.cpu().numpy()[counts:].reshape(-1)[:budget], w[kept.cpu().numpy()[0, 0]])


@pytest.mark.gpu
def test_evict_of_equal_weights_and_of_bad_tables():
    """All weights equal: the lowest tokens stay.  Pages that are not there: no access outside the pool."""
    import torch
    rng = np.random.default_rng(9)
    ref = R.RefCache(rng, 12, 2, 16, 64, "int8")
    ref.weight[:] = 0.0
    cache = R.to_device(ref, torch, B)
    pages, new_pages = np.arange(6, dtype=np.int32).reshape(1, 6), np.array([[8, 9, 10]], np.int32)
    kept, new_len = torch.empty(1, 2, 40, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_EVICT, cache, 1, 6), dtype=torch.uint8, device="cuda")
    B.fcp_cache_evict(cache, dev(pages), dev([90]), dev(new_pages), 40, 3, 5, kept, new_len, scratch)
    assert kept.cpu().numpy().tolist() == [[list(range(35)) + list(range(85, 90))] * 2]
    ref.evict(pages, [90], new_pages, 40, 3, 5)
    R.check_content(cache, ref)
    for lens, old, new in (([-3], pages, new_pages), ([10 ** 9], np.array([[0, -1, 99, 3, 4, 5]]), new_pages), ([90], pages, np.array([[-1, 10 ** 9, 11]]))):
        B.fcp_cache_evict(cache, dev(old), dev(lens), dev(new), 40, 3, 5, kept, new_len, scratch)
        assert int(new_len[0]) == min(max(lens[0], 0), 40)
    k, _, _, _, _ = R.from_device(cache)
    assert np.array_equal(k[:6], ref.k[:6]) and np.array_equal(k[6:8], ref.k[6:8])


def test_scales_that_would_vanish_are_refused():
    """softmax_scale times the least scale of a page must stay above 0, or a masked score, -inf, becomes NaN."""
    for op in ("attn", "weigh"):
        call = lambda v: getattr(Call(scale=v, n_seqs=0), op)()
        assert call(2.0 ** -33) == B.FCP_ERR_INVALID_ARG and call(float("inf")) == B.FCP_ERR_INVALID_ARG and call(-1.0) == B.FCP_ERR_INVALID_ARG
        assert call(2.0 ** -32) == 0 and call(1.0) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 40])
def test_least_scales_beside_masked_tokens(rows):
    """Pages of zeros (scale 2^-110) with the least softmax_scale: every seen token gets the same weight."""
    import torch
    P, D, n = 16, 64, 75
    pages = -(-n // P)
    z = lambda *s, dt=torch.int8: torch.zeros(*s, dtype=dt, device="cuda")
    cache = B.Cache(z(pages, 1, P, D), z(pages, 1, P // 16, D, 16), z(pages, 1, dt=torch.float32), z(pages, 1, dt=torch.float32), z(pages, 1, P, dt=torch.float32))
    cache.k_scale.fill_(2.0 ** -110), cache.v_scale.fill_(2.0 ** -110)
    q = np.ones((rows, 2, D))
    o, lse = run_attn(cache, q, np.array([0, rows]), [n], np.arange(pages, dtype=np.int32)[None], 2.0 ** -32, True)
    seen = n - rows + 1 + np.arange(rows)
    # the sum of n ones is exact; its logarithm is off by a few steps of itself
    assert (o == 0).all() and (np.abs(lse - np.log(seen)) <= np.log(seen) * 8 * 2.0 ** -24).all()
    want = sum(2.0 / s * (np.arange(pages * P) < s) for s in seen)
    got = cache.weight.double().cpu().numpy().reshape(-1)
    assert (np.abs(got - want) <= want * (2 * rows + 40) * 2.0 ** -24).all()


@pytest.mark.gpu
@pytest.mark.parametrize("news", [[1, 1, 1], [50, 60, 70]])
def test_rows_of_several_sequences_are_not_worked(news):
    """cu_seqlens that falls: more places than the host counted, so nothing is computed and nothing is written, in scratch neither."""
    import torch
    kv_len = [150, 130, 140]
    ref, cache, pages, cu, q, scale = attn_case(32, 64, 4, 2, kv_len, news, "int8")
    total = int(cu[-1])
    for bad in ([0, total, 0, total], [0, 2, 1, total], [total, 0, 0, 0], [0, 2147483647, -2147483648, total]):
        for which, weigh in ((B.FCP_SCRATCH_CACHE_ATTN, False), (B.FCP_SCRATCH_CACHE_WEIGH, True)):
            n = B.fcp_cache_scratch_bytes(which, cache, 3, pages.shape[1], total, 4)
            scratch = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
            o, lse = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((4, total), 7.0, device="cuda")
            B.fcp_cache_attn(cache, dev_bf16(q), dev(bad), dev(kv_len), dev(pages), scale, o, lse, scratch[:n], weigh=weigh)
            assert (o == 7).all() and (lse == 7).all() and (scratch[n:] == 77).all()
        B.fcp_cache_weigh(cache, dev_bf16(q), torch.zeros(4, total, device="cuda"), dev(bad), dev(kv_len), dev(pages), scale)
        assert np.array_equal(R.check_content(cache, ref), ref.weight.astype(np.float32))
    # and the same call with good ones works
    check_attn(run_attn(cache, q, cu, kv_len, pages, scale, False), ref.attn(q, cu, kv_len, pages, scale))


@pytest.mark.gpu
@pytest.mark.parametrize("news", [[1, 1], [3, 2], [40, 65]])
def test_queries_that_are_slices_of_wider_rows(news):
    """Rows of the fused projection's output: bit for bit the results of rows that lie together."""
    import torch
    kv_len = [300, 90]
    _, cache, pages, cu, q, scale = attn_case(64, 128, 6, 2, kv_len, news, "e4m3")
    n = int(cu[-1])
    wide = torch.full((n, 6 * 128 + 520), float("nan"), dtype=torch.bfloat16, device="cuda")
    sliced = wide[:, 8: 8 + 768].unflatten(1, (6, 128))
    sliced.copy_(dev_bf16(q))
    out = []
    for x in (dev_bf16(q), sliced):
        cache.weight.zero_()
        o, lse = torch.empty(n, 6, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(6, n, device="cuda")
        scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_WEIGH, cache, 2, pages.shape[1], n, 6), dtype=torch.uint8, device="cuda")
        B.fcp_cache_attn(cache, x, dev(cu), dev(kv_len), dev(pages), scale, o, lse, scratch, weigh=True)
        first = cache.weight.clone()
        B.fcp_cache_weigh(cache, x, lse, dev(cu), dev(kv_len), dev(pages), scale)
        out.append((o, lse, first, cache.weight.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_past_the_32nd_bit(fmt):
    """The last pages of a pool whose keys take more than 2^32 bytes: bit for bit what the same pages give in a small pool."""
    import torch
    P, D, hkv, hq, kv_len = 128, 128, 8, 8, [700, 260]
    dt = torch.int8
    used = 16
    n_big = (1 << 32) // (P * D * hkv) + used
    view = lambda t: t.view(torch.float8_e4m3fn) if fmt == "e4m3" else t
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = lambda n, h: torch.randn(n, h, D, generator=g, device="cuda").to(torch.bfloat16)
    cu, cu1 = np.array([0, 700, 960]), np.array([0, 70, 71])
    k, v, q = rows(960, hkv), rows(960, hkv), rows(71, hq)
    lse_in = torch.full((hq, 71), 6.0, device="cuda")
    results = []
    for n in (used, n_big):
        at = n - used
        mk = lambda *s: view(torch.empty(*s, dtype=dt, device="cuda"))
        cache = B.Cache(mk(n, hkv, P, D), mk(n, hkv, P // 16, D, 16), torch.empty(n, hkv, device="cuda"), torch.empty(n, hkv, device="cuda"), torch.empty(n, hkv, P, device="cuda"))
        for t in (cache.k, cache.v, cache.weight):
            (t.view(torch.int8) if t.element_size() == 1 else t)[at:].zero_()
        cache.k_scale[at:].fill_(1.0), cache.v_scale[at:].fill_(1.0)
        pages = dev(np.array([[5, 0, 3, 7, 1, 9], [2, 8, 4, -1, -1, -1]], np.int32) + at * np.array([[1] * 6, [1, 1, 1, 0, 0, 0]], np.int32))
        new_pages = dev(np.array([[12, 10], [15, 6]], np.int32) + at)
        B.fcp_cache_append(cache, k, v, dev(cu), dev(kv_len), pages)
        got = []
        for rows_cu, x in ((cu1, q), (np.array([0, 1, 2]), q[:2])):
            m = x.shape[0]
            o, lse = torch.empty(m, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(hq, m, device="cuda")
            scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_WEIGH, cache, 2, 6, m, hq), dtype=torch.uint8, device="cuda")
            B.fcp_cache_attn(cache, x, dev(rows_cu), dev(kv_len), pages, 0.09, o, lse, scratch, weigh=True)
            got += [o, lse]
        B.fcp_cache_weigh(cache, q, lse_in, dev(cu1), dev(kv_len), pages, 0.09)
        kept, new_len = torch.empty(2, hkv, 200, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
        scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_EVICT, cache, 2, 6), dtype=torch.uint8, device="cuda")
        B.fcp_cache_evict(cache, pages, dev(kv_len), new_pages, 200, 4, 30, kept, new_len, scratch)
        got += [kept, new_len, cache.k_scale[at:].clone(), cache.v_scale[at:].clone(), cache.weight[at:].clone()]
        got += [t.view(torch.int8)[at:].clone() for t in (cache.k, cache.v)]
        results.append(got)
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert float(results[0][8].sum()) > 100 and not torch.isnan(results[0][0].float()).any()


SEVERAL = [  # P, D, hq, hkv, kv_len, news: 17 to 32 rows of a KV head per sequence on average, more and fewer in some
    (16, 64, 8, 2, [100, 37], [7, 4]), (64, 128, 16, 1, [1300], [2]), (32, 128, 8, 1, [2500, 40, 0, 700], [3, 2, 1, 4]), (128, 64, 24, 1, [5, 900], [1, 1]),
    (64, 128, 8, 2, [150, 64, 1], [15, 3, 1]), (16, 128, 8, 8, [600, 19, 5], [32, 21, 9]), (32, 64, 40, 8, [1100, 1090], [5, 6])]


@pytest.mark.gpu
@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news", SEVERAL)
def test_attention_of_several_tokens(P, D, hq, hkv, kv_len, news, fmt, weigh):
    assert 16 < sum(news) * hq / hkv / len(news) <= 32
    ref, cache, pages, cu, q, scale = attn_case(P, D, hq, hkv, kv_len, news, fmt, seed=7)
    got = run_attn(cache, q, cu, kv_len, pages, scale, weigh)
    want = ref.attn(q, cu, kv_len, pages, scale)
    eps = check_attn(got, want)
    w = R.check_content(cache, ref)
    if weigh:
        check_weight(w, ref.weight, want[2], eps, max(news) * hq // hkv)
    else:
        assert np.array_equal(w, ref.weight.astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [90, 1500])
@pytest.mark.parametrize("news", [1, 5, 12])
def test_nan_values_reach_only_the_rows_that_see_them(D, n, news):
    """NaN in values of the last tokens, in several channels and tiles' waves, and past the last token; short tables, and long ones whose items are divided."""
    ref, cache, pages, cu, q, scale = attn_case(64, D, 4, 2, [n, n - 7], [news, news], "e4m3", seed=3)
    for s, length in ((0, n), (1, n - 7)):
        ref.v[pages[s, (length - 1) // 64], :, (length - 1) % 64 + 1:] = 127
        for back, head, channel in ((1, 0, 3), (2, 1, 17), (1, 1, 40), (5, 1, 40), (11, 0, 63)):
            t = length - back
            ref.v[pages[s, t // 64], head, t % 64, channel] = 255 if back % 2 else 127
    import torch
    cache = R.to_device(ref, torch, B)
    got = run_attn(cache, q, cu, [n, n - 7], pages, scale, False)
    want = ref.attn(q, cu, [n, n - 7], pages, scale)
    assert np.isnan(want[0]).any() and (news == 1 or not np.isnan(want[0][:, 0, 3]).all())
    check_attn(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("news", [1, 5])
@pytest.mark.parametrize("hkv", [1, 4])
def test_nothing_is_written_past_scratch(news, hkv):
    """Scratch of exactly the size that is asked for, in a longer tensor whose other bytes stay."""
    import torch
    kv_len = [1000, 64, 1, 0, 1999]
    ref, cache, pages, cu, q, scale = attn_case(32, 64, 4, hkv, kv_len, [news] * 5, "int8", seed=5)
    for which, weigh in ((B.FCP_SCRATCH_CACHE_ATTN, False), (B.FCP_SCRATCH_CACHE_WEIGH, True)):
        n = B.fcp_cache_scratch_bytes(which, cache, 5, pages.shape[1], q.shape[0], 4)
        scratch = torch.full((n + 65536,), 77, dtype=torch.uint8, device="cuda")
        o, lse = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda"), torch.empty(4, q.shape[0], device="cuda")
        B.fcp_cache_attn(cache, dev_bf16(q), dev(cu), dev(kv_len), dev(pages), scale, o, lse, scratch[:n], weigh=weigh)
        assert (scratch[n:] == 77).all()
        check_attn((o.double().cpu().numpy(), lse.double().cpu().numpy()), ref.attn(q, cu, kv_len, pages, scale))


@pytest.mark.gpu
@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news", [   # 33 to 64 rows of a KV head per sequence on average
    (64, 128, 40, 8, [600, 90], [10, 9]), (16, 64, 6, 2, [1200], [20]), (32, 128, 16, 1, [2300, 77, 5], [7, 2, 1]), (128, 64, 4, 4, [70, 1500], [64, 33])])
def test_attention_of_tens_of_rows(P, D, hq, hkv, kv_len, news, fmt, weigh):
    assert 32 < sum(news) * hq / hkv / len(news) <= 64
    ref, cache, pages, cu, q, scale = attn_case(P, D, hq, hkv, kv_len, news, fmt, seed=9)
    got = run_attn(cache, q, cu, kv_len, pages, scale, weigh)
    want = ref.attn(q, cu, kv_len, pages, scale)
    eps = check_attn(got, want)
    w = R.check_content(cache, ref)
    if weigh:
        check_weight(w, ref.weight, want[2], eps, max(news) * hq // hkv)
    else:
        assert np.array_equal(w, ref.weight.astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [90, 1500])
def test_nan_values_among_tens_of_rows(D, n):
    import torch
    ref, cache, pages, cu, q, scale = attn_case(64, D, 4, 2, [n, n - 7], [24, 24], "e4m3", seed=3)
    for s, length in ((0, n), (1, n - 7)):
        for back, head, channel in ((1, 0, 3), (2, 1, 17), (5, 1, 40), (21, 0, 63)):
            t = length - back
            ref.v[pages[s, t // 64], head, t % 64, channel] = 255
    cache = R.to_device(ref, torch, B)
    got = run_attn(cache, q, cu, [n, n - 7], pages, scale, False)
    want = ref.attn(q, cu, [n, n - 7], pages, scale)
    assert np.isnan(want[0]).any() and not np.isnan(want[0][0]).any()
    check_attn(got, want)
