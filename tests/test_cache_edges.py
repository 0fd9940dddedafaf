"""The paged 8-bit cache at the edges of what it takes: what unused pages hold, the ends of the range of scales and scores, queries that are not finite, limits."""
import numpy as np
import pytest

import cache_ref as R
from paper_2602_21788_amd import binding as B
from test_cache import FORMATS, Call, attn_case, check_attn, dev, dev_bf16, run_attn


# ---- CPU ------------------------------------------------------------------------------------------------------------------------------------
def test_launches_of_too_many_threads_are_refused_before_any_device_work():
    no = B.FCP_ERR_UNSUPPORTED
    assert Call(page_tokens=16, n_rows=1 << 28).append() == no and Call(page_tokens=16, n_rows=2 ** 31 - 1, n_seqs=1).append() == no
    assert Call(n_seqs=1 << 20).evict() == no and b"2^22" in B.lib().fcp_last_error()
    assert Call(hkv=1, page_tokens=16, n_seqs=1 << 20, max_pages=16, max_new=16, budget=256).evict() == no
    p = (B.RotaryPart * 1)()
    p[0].x = p[0].y = p[0].pos = Call.fake
    p[0].x_row = p[0].y_row = p[0].x_head = p[0].y_head = 1024
    p[0].rows, p[0].heads = 1 << 24, 1
    assert B.lib().fcp_rotary(p, 1, Call.fake, 1024, 1024, 0, 1.0, 0, None) == no and b"2^24" in B.lib().fcp_last_error()


def test_places_that_a_step_would_take_past_32_bits_are_refused():
    """A block of the weights' kernel steps 1024 places at a time, past the last one too: 2^31 - 128 places and their likes were let through."""
    call = lambda op, pages, heads: getattr(Call(hkv=heads, hq=heads, q_row=128 * heads, n_seqs=1, tq=1, max_pages=pages, bytes=0), op)()
    for pages, heads in (((1 << 24) - 5, 128), ((1 << 23) - 5, 256)):
        assert call("attn", pages, heads) == call("weigh", pages, heads) == B.FCP_ERR_UNSUPPORTED, (pages, heads)
    assert call("attn", (1 << 20) - 5, 2048) == B.FCP_ERR_CAPACITY             # 2^31 - 2048: scratch is what is missing


def test_scratch_is_refused_where_the_call_is():
    f = B.fcp_cache_scratch_bytes
    sizes = lambda which, n_seqs, max_pages, tq=4, hq=16, **c: f(which, Call(**c).c, n_seqs, max_pages, tq, hq)
    which = (B.FCP_SCRATCH_CACHE_ATTN, B.FCP_SCRATCH_CACHE_WEIGH, B.FCP_SCRATCH_CACHE_EVICT)
    for w in which:
        for n_seqs, max_pages in (((1 << 20) + 1, 4), (4, (1 << 24) + 1), (-1, 4), (4, -1)):
            with pytest.raises(B.FcpError):
                sizes(w, n_seqs, max_pages)
        assert sizes(w, 4, 1 << 24, hkv=1, hq=1) > 0 and sizes(w, 0, 4) > 0
    for w in which[:2]:
        for n_seqs, max_pages, tq, hq in ((4, 4, 1 << 27, 16), (1 << 20, 1 << 10, 4, 16), (4, 4, 4, 6)):
            with pytest.raises(B.FcpError):
                sizes(w, n_seqs, max_pages, tq, hq)
            assert Call(n_seqs=n_seqs, max_pages=max_pages, tq=tq, hq=hq, q_row=128 * hq).attn() == B.FCP_ERR_UNSUPPORTED
        assert sizes(w, 4, 4, tq=0) > 0
    with pytest.raises(B.FcpError):
        sizes(which[2], 1 << 20, 1)


# ---- GPU ------------------------------------------------------------------------------------------------------------------------------------
def check_weights(got, before, W, eps, rows):
    """As test_cache.check_weight where the sums are finite; elsewhere the same NaN and infinity."""
    want = before + W
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine) and np.array_equal(got[~fine], want[~fine], equal_nan=True)
    tol = W[fine] * (2 * eps[np.isfinite(eps)].max() + 1e-6) + want[fine] * (rows + 2) * 2.0 ** -24 + 1e-30
    assert (np.abs(got[fine] - want[fine]) <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news", [   # rows of a KV head per sequence on average: up to 16, 32, 64, more; whole and divided items
    (16, 64, 4, 2, [150, 70], [1, 2]), (32, 128, 8, 2, [1500, 40], [6, 6]), (16, 64, 4, 2, [150, 70], [20, 20]), (32, 128, 8, 2, [1500, 40], [16, 10]),
    (16, 64, 4, 2, [150, 70], [50, 60]), (64, 128, 4, 1, [1500, 129], [40, 40]), (128, 128, 4, 2, [65], [65])])
def test_scales_of_unused_pages_are_not_looked_at(P, D, hq, hkv, kv_len, news, fmt, bad):
    """Nobody has to fill the scales of pages that hold no token: NaN and infinity there reach nothing.  Page 0 is unused, and a page in the middle is missing."""
    import torch
    ref, _, pages, cu, q, scale = attn_case(P, D, hq, hkv, kv_len, news, fmt, seed=11)
    grown = R.RefCache(np.random.default_rng(0), ref.n_pages + 1, hkv, P, D, fmt)
    for name in ("k", "v", "k_e", "v_e", "weight"):
        getattr(grown, name)[1:] = getattr(ref, name)
    pages = np.where(pages >= 0, pages + 1, -1).astype(np.int32)
    if (pages[0] >= 0).sum() > 2:
        pages[0, 1] = -1
    cache = R.to_device(grown, torch, B)
    unused = torch.from_numpy(np.setdiff1d(np.arange(grown.n_pages), pages)).cuda()
    assert 0 in unused
    cache.k_scale[unused], cache.v_scale[unused] = bad, bad
    for weigh in (False, True):
        got = run_attn(cache, q, cu, kv_len, pages, scale, weigh)
        want = grown.attn(q, cu, kv_len, pages, scale)
        assert np.isfinite(want[0]).all()
        eps = check_attn(got, want)
    check_weights(R.from_device(cache)[4], grown.weight, want[2], eps, max(news) * hq // hkv)


@pytest.mark.gpu
@pytest.mark.parametrize("P,D", [(16, 64), (64, 128)])
@pytest.mark.parametrize("far", [17, 18, 60, 119])
@pytest.mark.parametrize("fmt", FORMATS)
def test_eviction_keeps_zeros_of_pages_of_great_scales(fmt, far, P, D):
    """Tokens of nothing but zeros from a page whose scale is 2^far: alone in a new page, whose scale is the least, and beside tokens of the least magnitudes."""
    import torch
    rng = np.random.default_rng(far)
    ref = R.RefCache(rng, 10, 2, P, D, fmt)
    pages, new_pages = np.array([[0, 1, 2], [3, 4, 5]], np.int32), np.array([[6], [7]], np.int32)
    kv_len, budget = [3 * P, 3 * P], P
    ref.weight[:] = 0
    for codes, es in ((ref.k, ref.k_e), (ref.v, ref.v_e)):
        es[[0, 3]], es[1] = far, -108
        codes[0, :, ::2] = codes[3] = 0
        codes[3, :, 1, 5] = 0 if fmt == "int8" else 128          # minus zero
    ref.weight[0, :, ::2], ref.weight[1, :, ::2], ref.weight[3] = 2, 1, 1
    cache = R.to_device(ref, torch, B)
    kept, new_len = torch.empty(2, 2, budget, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_EVICT, cache, 2, 3), dtype=torch.uint8, device="cuda")
    B.fcp_cache_evict(cache, dev(pages), dev(kv_len), dev(new_pages), budget, 0, 0, kept, new_len, scratch)
    want_kept, _ = ref.evict(pages, kv_len, new_pages, budget, 0, 0)
    assert np.array_equal(kept.cpu().numpy(), want_kept) and ref.k_e[7, 0] == R.LEAST and ref.k_e[6, 0] < -90
    R.check_content(cache, ref)


MANY = [  # P, D, hq, hkv, kv_len, news of calls of fcp_cache_weigh
    (64, 128, 4, 4, [100], [100]), (16, 64, 8, 2, [70, 130], [70, 130]), (32, 128, 6, 2, [300, 20, 90], [40, 20, 1]), (128, 64, 2, 2, [1000], [3]), (64, 128, 3, 1, [200], [17])]


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news", MANY)
def test_weights_of_queries_that_are_not_finite(P, D, hq, hkv, kv_len, news, bad):
    """Such a row reaches the weights of the tokens that it sees and no others."""
    import torch
    ref, cache, pages, cu, q, scale = attn_case(P, D, hq, hkv, kv_len, news, "int8", seed=21)
    _, LSE, _, _, units = ref.attn(q, cu, kv_len, pages, scale)
    lse = LSE.astype(np.float32)
    q[0, 0, 3] = bad
    B.fcp_cache_weigh(cache, dev_bf16(q), torch.from_numpy(lse).cuda(), dev(cu), dev(kv_len), dev(pages), scale)
    with np.errstate(all="ignore"):
        W = ref.attn(q, cu, kv_len, pages, scale, lse_in=lse.astype(np.float64))[2]
    eps = (units + 8 * np.abs(LSE) + 16) * 2.0 ** -24
    check_weights(R.from_device(cache)[4], ref.weight, W, eps, max(news) * hq // hkv)


@pytest.mark.gpu
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news", MANY)
def test_weights_of_rows_whose_sum_is_nan_or_of_nothing(P, D, hq, hkv, kv_len, news):
    """A row whose LSE is -inf adds nothing, whatever its query holds; one whose LSE is NaN reaches the tokens that it sees and no others."""
    import torch
    ref, cache, pages, cu, q, scale = attn_case(P, D, hq, hkv, kv_len, news, "e4m3", seed=22)
    _, LSE, _, _, units = ref.attn(q, cu, kv_len, pages, scale)
    lse, n = LSE.astype(np.float32), q.shape[0]
    given, seen_by, sums = q.copy(), q.copy(), lse.astype(np.float64)
    for row, value in ((n - 1, np.nan), (n // 2, np.inf)):
        given[row], seen_by[row], lse[:, row], sums[:, row] = value, 0, -np.inf, np.inf          # (exp(score - inf) is 0)
    lse[0, 0] = sums[0, 0] = np.nan
    B.fcp_cache_weigh(cache, dev_bf16(given), torch.from_numpy(lse).cuda(), dev(cu), dev(kv_len), dev(pages), scale)
    W = ref.attn(seen_by, cu, kv_len, pages, scale, lse_in=sums)[2]
    eps = (units + 8 * np.abs(LSE) + 16) * 2.0 ** -24
    check_weights(R.from_device(cache)[4], ref.weight, W, eps, max(news) * hq // hkv)


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news", MANY + [(16, 64, 4, 2, [90, 33], [3, 2]), (64, 128, 2, 1, [1500], [6]), (32, 64, 1, 1, [70, 200], [5, 9])])
def test_attention_that_weighs_queries_that_are_not_finite(P, D, hq, hkv, kv_len, news, bad):
    """A row whose query is not finite spoils its own output and sum, and the weights of the tokens that it sees; nothing else."""
    import torch
    ref, cache, pages, cu, q, scale = attn_case(P, D, hq, hkv, kv_len, news, "int8", seed=23)
    q[0, 0] = 0                                            # (the reference's row: what it adds lies on the tokens that are left out below)
    want = ref.attn(q, cu, kv_len, pages, scale)
    q[0, 0, 3] = bad
    o, lse = run_attn(cache, q, cu, kv_len, pages, scale, True)
    assert bad == np.inf or (np.isnan(o[0, 0]).all() and np.isnan(lse[0, 0]))
    o[0, 0], lse[0, 0] = want[0][0, 0], want[1][0, 0]
    eps = check_attn((o, lse), want)
    got, mine = R.from_device(cache)[4].astype(np.float64), np.zeros(ref.weight.shape, bool)
    for t in range(kv_len[0] - news[0] + 1):
        mine[pages[0, t // P], 0, t % P] = True
    assert bad == np.inf or np.isnan(got[mine]).all()
    got[mine] = (ref.weight + want[2])[mine]
    check_weights(got, ref.weight, want[2], eps, max(news) * hq // hkv)


PARTS = [  # P, D, hq, hkv, kv_len, news, softmax scale: up to 32 rows of a KV head per sequence on average; items whole, and (more than 2048 tokens in the table, or weights) divided
    (16, 64, 4, 2, [100, 37], [1, 1], 0.125), (64, 128, 8, 1, [300, 90], [1, 2], 0.09), (32, 128, 4, 4, [2500], [1], 0.3), (64, 64, 8, 2, [2300, 3000], [2, 4], 0.4),
    (16, 64, 8, 2, [100, 37], [7, 4], 0.125), (64, 128, 24, 1, [200], [1], 0.09), (32, 128, 8, 1, [2500], [4], 0.3)]


def part_bound(q, ref, want, kv_len, news, bits):
    """What O may be off by: half a step of bf16 of itself; of sum p |v| the `bits` that the probabilities in the product have, twice what a score may be off by, and the roundings of the sums of
    numerator and denominator.  On its way through both a term meets at most 16 additions for each tile of its wave, 64 in a product and 64 where waves and pieces are joined."""
    O, LSE, _, absv, units = want
    eps = (units + 8 * np.abs(LSE) + 16) * 2.0 ** -24
    sums = 2 * (max(kv_len) // 16 + 128) * 2.0 ** -24
    return absv * (2.0 ** -bits + 2 * eps.T[..., None] + sums) + np.abs(O) * 2.0 ** -8 + 1e-30


def parts_case(P, D, hq, hkv, kv_len, news, scale, fmt):
    assert sum(news) * hq / hkv / len(news) <= 32
    ref, cache, pages, cu, q, scale = attn_case(P, D, hq, hkv, kv_len, news, fmt, seed=31, scale=scale)
    return ref, cache, pages, cu, q, scale, ref.attn(q, cu, kv_len, pages, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news,scale", PARTS)
def test_probabilities_of_few_rows_have_two_parts(P, D, hq, hkv, kv_len, news, scale, fmt, weigh):
    """Two bf16 parts: what a part leaves is at most 2^-8 of what it is a part of."""
    ref, cache, pages, cu, q, scale, want = parts_case(P, D, hq, hkv, kv_len, news, scale, fmt)
    o, _ = run_attn(cache, q, cu, kv_len, pages, scale, weigh)
    assert (np.abs(o - want[0]) <= part_bound(q, ref, want, kv_len, news, 16)).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("P,D,hq,hkv,kv_len,news,scale", PARTS)
def test_the_bound_tells_one_part_from_two(P, D, hq, hkv, kv_len, news, scale, fmt, monkeypatch):
    """On the CPU, exactly but for the probabilities: in two parts they are within the bound, in one they are not."""
    monkeypatch.setattr(R, "to_device", lambda *a: None)
    ref, _, pages, cu, q, scale, want = parts_case(P, D, hq, hkv, kv_len, news, scale, fmt)

    def bf16(x):
        u = np.asarray(x, np.float32).view(np.uint32)
        return ((u + 0x7fff + ((u >> 16) & 1)) & np.uint32(0xffff0000)).view(np.float32).astype(np.float64)

    off = {1: np.zeros(want[0].shape), 2: np.zeros(want[0].shape)}
    for s, n in enumerate(kv_len):
        for h in range(hq):
            K, V = (ref.rows(w, pages[s], n, h // (hq // hkv))[0] for w in "kv")
            for i in range(news[s]):
                x = scale * (K @ q[cu[s] + i, h])
                e = np.exp(x - x[: n - news[s] + i + 1].max()) * (np.arange(n) <= n - news[s] + i)
                one = bf16(e)
                for parts, p in ((1, one), (2, one + bf16(e - one))):
                    off[parts][cu[s] + i, h] = bf16(p @ V / e.sum()) - want[0][cu[s] + i, h]
    bound = part_bound(q, ref, want, kv_len, news, 16)
    assert (np.abs(off[2]) <= bound).all() and (np.abs(off[1]) > bound).any()


@pytest.mark.gpu
def test_eviction_with_a_budget_of_the_last_32_bit_number():
    """A budget far above what the tables can hold keeps everything; the list's end is -1 to the last place."""
    import torch
    ref = R.RefCache(np.random.default_rng(3), 5, 1, 16, 64, "int8")
    cache = R.to_device(ref, torch, B)
    pages, new_pages, budget = np.array([[0, 1]], np.int32), np.array([[3, 2]], np.int32), 2 ** 31 - 1
    kept, new_len = torch.zeros(1, 1, budget, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_EVICT, cache, 1, 2), dtype=torch.uint8, device="cuda")
    B.fcp_cache_evict(cache, dev(pages), dev([21]), dev(new_pages), budget, 4, 8, kept, new_len, scratch)
    assert int(new_len[0]) == 21 and kept[0, 0, :21].tolist() == list(range(21))
    assert all(bool((x == -1).all()) for x in kept[0, 0, 21:].split(1 << 28))
    ref.evict(pages, [21], new_pages, 24, 4, 8)
    R.check_content(cache, ref)


@pytest.mark.gpu
def test_eviction_with_a_long_table_of_new_pages():
    """Only as many entries as the budget fills are launched for."""
    import torch
    ref = R.RefCache(np.random.default_rng(4), 9, 2, 16, 64, "e4m3")
    cache = R.to_device(ref, torch, B)
    pages, new_pages, kv_len = np.array([[0, 1, 2], [3, 4, -1]], np.int32), np.full((2, 1 << 23), -1, np.int32), [41, 19]
    new_pages[:, :2] = [[8, 5], [6, 7]]
    kept, new_len = torch.empty(2, 2, 20, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_EVICT, cache, 2, 3), dtype=torch.uint8, device="cuda")
    B.fcp_cache_evict(cache, dev(pages), dev(kv_len), dev(new_pages), 20, 1, 4, kept, new_len, scratch)
    want_kept, want_len = ref.evict(pages, kv_len, new_pages, 20, 1, 4)
    assert np.array_equal(kept.cpu().numpy(), want_kept) and np.array_equal(new_len.cpu().numpy(), want_len)
    R.check_content(cache, ref)
