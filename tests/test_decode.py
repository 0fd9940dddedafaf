"""Prompts, new tokens and eviction together: the decoder against attention in 64 bits over what its cache holds, token for token."""
import numpy as np
import pytest

import cache_ref as R
from paper_2602_21788_amd import binding as B


def bf16_rows(torch, g, n, h, D):
    return torch.randn(n, h, D, generator=g, device="cuda").to(torch.bfloat16)


def held(dec, fmt):
    """The cache's content as the reference's."""
    k, v, ks, vs, w = R.from_device(dec.cache)
    ref = object.__new__(R.RefCache)
    ref.P, ref.D, ref.hkv, ref.fmt, ref.n_pages = dec.P, dec.D, dec.hkv, fmt, k.shape[0]
    ref.k, ref.v, ref.k_e, ref.v_e, ref.weight = k, v, np.log2(ks).astype(int), np.log2(vs).astype(int), w.astype(np.float64)
    return ref


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,P,D,hq,hkv", [("e4m3", 64, 128, 8, 2), ("int8", 16, 64, 4, 4)])
def test_prompts_tokens_and_eviction(fmt, P, D, hq, hkv):
    import torch
    from paper_2602_21788_amd.decode import CacheDecoder
    g = torch.Generator(device="cuda").manual_seed(1)
    lens = [150, 3, 0, 64]
    dec = CacheDecoder(4, 64, 24, hq, hkv, D, page_tokens=P, fmt=fmt)
    n = sum(lens)
    q, k, v = bf16_rows(torch, g, n, hq, D), bf16_rows(torch, g, n, hkv, D), bf16_rows(torch, g, n, hkv, D)
    before = held(dec, fmt)
    o, lse = dec.prefill(q, k, v, lens)
    f64 = lambda t: t.double().cpu().numpy()
    cu = np.concatenate([[0], np.cumsum(lens)])
    # the cache holds the prompts' rotated keys and values, and the weights of the prompts' own attention
    before.append(f64(k), f64(v), cu, dec.kv_len, dec.pages)
    w = R.check_content(dec.cache, before)
    _, _, want, _, units = before.attn(f64(q), cu, dec.kv_len, dec.pages, dec.scale, lse_in=f64(lse))
    assert np.abs(w - want).max() <= 1e-5 * max(lens) and (want > 0).any()

    def check_step(news):
        rows = sum(news)
        q, k, v = bf16_rows(torch, g, rows, hq, D), bf16_rows(torch, g, rows, hkv, D), bf16_rows(torch, g, rows, hkv, D)
        ref = held(dec, fmt)
        o, lse = dec.step(q, k, v, news)
        cu = np.concatenate([[0], np.cumsum(news)])
        ref.append(f64(k), f64(v), cu, dec.kv_len, dec.pages)
        O, LSE, W, absv, units = ref.attn(f64(q), cu, dec.kv_len, dec.pages, dec.scale)
        eps = (units + 8 * np.abs(LSE) + 16) * 2.0 ** -24
        assert (np.abs(f64(lse) - LSE) <= eps).all()
        assert (np.abs(f64(o) - O) <= absv * (2.0 ** -8 + 2 * eps.T[..., None]) + np.abs(O) * 2.0 ** -8 + 1e-30).all()
        w = R.check_content(dec.cache, ref)
        assert (np.abs(w - ref.weight - W) <= 1e-4 * W + (ref.weight + W) * 2.0 ** -22 + 1e-30).all()

    for news in ([1, 1, 1, 1], [1, 1, 0, 1], [0, 7, 2, 1]):
        check_step(news)
    assert dec.next_pos.tolist() == [152, 12, 3, 67]
    ref = held(dec, fmt)
    lens, pages, free = dec.kv_len.copy(), dec.pages.copy(), len(dec.free)
    kept = dec.evict(60, n_first=2, n_recent=16)
    want_kept, want_len = ref.evict(pages, lens, dec.pages, 60, 2, 16)
    assert np.array_equal(kept.cpu().numpy(), want_kept) and np.array_equal(dec.kv_len, want_len)
    assert len(dec.free) == free + (pages >= 0).sum() - (dec.pages >= 0).sum()
    assert dec.next_pos.tolist() == [152, 12, 3, 67]
    for news in ([1, 1, 1, 1], [2, 0, 1, 30]):
        check_step(news)
    dec.close(0)
    assert dec.kv_len[0] == 0 and (dec.pages[0] == -1).all()
    check_step([5, 1, 1, 1])


@pytest.mark.gpu
def test_the_decoder_says_when_pages_are_short():
    import torch
    from paper_2602_21788_amd.decode import CacheDecoder
    g = torch.Generator(device="cuda").manual_seed(2)
    dec = CacheDecoder(2, 6, 4, 2, 2, 64, page_tokens=16)
    rows = lambda n: (bf16_rows(torch, g, n, 2, 64) for _ in range(3))
    dec.prefill(*rows(64), [40, 24])
    with pytest.raises(MemoryError):
        dec.step(*rows(30), [30, 0])
    with pytest.raises(MemoryError):
        dec.evict(32, 1, 1)
    assert dec.kv_len.tolist() == [40, 24]
    dec.close(1)
    dec.evict(16, 1, 4)
    assert dec.kv_len.tolist() == [16, 0] and len(dec.free) == 5
    with pytest.raises(ValueError):
        dec.prefill(*rows(4), [2, 2])


@pytest.mark.gpu
def test_refusals_change_nothing():
    import torch
    from paper_2602_21788_amd.decode import CacheDecoder
    dec = CacheDecoder(2, 8, 4, 4, 2, 64, page_tokens=16)
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = lambda n, h: bf16_rows(torch, g, n, h, 64)
    dec.prefill(rows(50, 4), rows(50, 2), rows(50, 2), [40, 10])
    free, lens, pages = list(dec.free), dec.kv_len.copy(), dec.pages.copy()
    for call in (lambda: dec.evict(20, n_first=4, n_recent=64), lambda: dec.evict(0, 0, 0), lambda: dec.evict(20, -1, 4),
                 lambda: dec.step(rows(3, 4), rows(3, 2), rows(3, 2), [1, 1]), lambda: dec.step(rows(1, 4), rows(1, 2), rows(1, 2), [2, -1]),
                 lambda: dec.step(rows(1, 4), rows(1, 2), rows(1, 2), [1]), lambda: dec.prefill(rows(1, 4), rows(1, 2), rows(1, 2), [1, 0])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(MemoryError):
        dec.step(rows(90, 4), rows(90, 2), rows(90, 2), [20, 70])
    assert dec.free == free and np.array_equal(dec.kv_len, lens) and np.array_equal(dec.pages, pages)


def state(dec):
    return list(dec.free), dec.kv_len.tolist(), dec.next_pos.tolist(), dec.pages.tolist()


@pytest.mark.gpu
def test_rows_of_another_kind_change_nothing():
    """Heads, channels, types and layouts that do not fit are refused before tokens are counted, pages taken or rows turned."""
    import torch
    from paper_2602_21788_amd.decode import CacheDecoder
    g = torch.Generator(device="cuda").manual_seed(6)
    rows = lambda n, h, d=64: bf16_rows(torch, g, n, h, d)
    good = rows(40, 4), rows(40, 2), rows(40, 2)
    for begun in (False, True):
        dec = CacheDecoder(2, 12, 6, 4, 2, 64, page_tokens=16)
        if begun:
            dec.prefill(*(x.clone() for x in good), [30, 10])
        before = state(dec)
        call = dec.step if begun else dec.prefill
        for at, heads in ((0, 4), (1, 2), (2, 2)):
            h = heads
            wide = rows(40, h + 1)
            for bad in (rows(40, h + 1), rows(40, h, 128), rows(40, h).float(), rows(40, h).cpu(), rows(40, h).reshape(40, -1), wide.transpose(1, 2), rows(39, h),
                        rows(40, h, 65)[:, :, 1:], torch.zeros(40 * (h * 64 + 4), dtype=torch.bfloat16, device="cuda").as_strided((40, h, 64), (h * 64 + 4, 64, 1))):
                args = [x.clone() for x in good]
                args[at] = bad
                with pytest.raises(ValueError):
                    call(*args, [15, 25])
                assert state(dec) == before
                assert all(torch.equal(x, y) for i, (x, y) in enumerate(zip(args, good)) if i != at)
        o, _ = call(*(x.clone() for x in good), [15, 25])
        assert torch.isfinite(o.float()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("where", ["_work", "fcp_rotary", "fcp_cache_append", "fcp_cache_attn", "fcp_cache_weigh", "fcp_cache_evict", "_to"])
def test_failures_leave_the_tables_as_they_were(where, monkeypatch):
    """Memory that is not there, or a call that fails: the decoder counts no token that it does not answer, and the next call works."""
    import torch
    from paper_2602_21788_amd import decode
    g = torch.Generator(device="cuda").manual_seed(7)
    rows = lambda n: (bf16_rows(torch, g, n, 4, 64), bf16_rows(torch, g, n, 2, 64), bf16_rows(torch, g, n, 2, 64))
    dec = decode.CacheDecoder(2, 24, 6, 4, 2, 64, page_tokens=16)
    calls = {"prefill": lambda: dec.prefill(*rows(40), [30, 10]), "step": lambda: dec.step(*rows(9), [4, 5]), "evict": lambda: dec.evict(20, 1, 4)}
    failing = {"fcp_rotary": ("prefill", "step"), "_to": ("prefill", "step", "evict"), "fcp_cache_append": ("prefill", "step"), "fcp_cache_attn": ("step",),
               "fcp_cache_weigh": ("prefill",), "fcp_cache_evict": ("evict",), "_work": ("step", "evict")}[where]
    for name, call in calls.items():
        if name in failing:
            before = state(dec)

            def fail(*a, **kw):
                raise torch.OutOfMemoryError("none left")

            with monkeypatch.context() as m:
                m.setattr(decode.B if where.startswith("fcp") else dec, where, fail)
                with pytest.raises(torch.OutOfMemoryError):
                    call()
            assert state(dec) == before, name
        call()
    lens, pages = dec.kv_len.tolist(), dec.pages
    assert lens == [20, 15] and sorted(dec.free + pages[pages >= 0].tolist()) == list(range(24))


@pytest.mark.gpu
def test_no_tokens_at_all():
    import torch
    from paper_2602_21788_amd.decode import CacheDecoder
    dec = CacheDecoder(2, 8, 4, 4, 2, 64, page_tokens=16)
    none = lambda h: torch.empty(0, h, 64, dtype=torch.bfloat16, device="cuda")
    for call in (dec.prefill, dec.step):
        o, lse = call(none(4), none(2), none(2), [0, 0])
        assert o.shape == (0, 4, 64) and lse.shape == (4, 0)
    assert dec.evict(16, 1, 4).eq(-1).all() and dec.kv_len.tolist() == [0, 0] and len(dec.free) == 8
