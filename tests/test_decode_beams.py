"""Beams over the cache, select -> fork -> rotary -> append -> attention together: every beam against a sequence of its own that was given the same rows one after the other."""
import numpy as np
import pytest

import cache_ref as R
from paper_2602_21788_amd import binding as B


def rows_of(cache, table, n, P, fmt):
    """Dequantised keys and values [n, hkv, D] of the first n tokens of a table, from the device."""
    k, v, ks, vs, _ = R.from_device(cache)
    out = []
    for codes, scales in ((k, ks), (v, vs)):
        x = R.decode(codes[table[: -(-n // P)]], fmt) * scales[table[: -(-n // P)]].astype(np.float64)[:, :, None, None]
        out.append(x.transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])[:n])
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("fmt, P, D, hq, hkv, beams, lens, rot, width", [
    ("e4m3", 64, 128, 8, 2, 4, [150, 3, 64], 128, 600), ("int8", 16, 64, 4, 4, 3, [33, 16, 1, 47], 0, 16), ("int8", 32, 64, 10, 2, 8, [100], 32, 3000), ("e4m3", 64, 128, 8, 2, 4, [150, 3, 64], 128, 16)])
def test_beams_are_sequences(fmt, P, D, hq, hkv, beams, lens, rot, width):
    """The cached tokens of every beam are, code for code, those of a sequence that was appended alone, whatever beams forked from each other; attention is that over its own table."""
    import torch
    from paper_2602_21788_amd.decode import BeamDecoder, CacheDecoder
    g = torch.Generator(device="cuda").manual_seed(P)
    rows = lambda n, h: torch.randn(n, h, D, generator=g, device="cuda").to(torch.bfloat16)
    n, steps, vocab = len(lens), 2 * P // 3 + 3, 500
    dec = BeamDecoder(n, beams, 200, width, hq, hkv, D, end_token=7, page_tokens=P, fmt=fmt, rot_dim=rot)
    alone = CacheDecoder(n * beams, 400, 16, hq, hkv, D, page_tokens=P, fmt=fmt, rot_dim=rot)
    q, k, v = rows(sum(lens), hq), rows(sum(lens), hkv), rows(sum(lens), hkv)
    again = [torch.cat([x[a: a + m] for a, m in zip(np.cumsum([0] + lens), lens) for _ in range(beams)]).contiguous() for x in (q, k, v)]
    dec.prefill(q, k, v, lens)
    # the rows of every step, and of every beam at the end the rows on its path
    given, paths = [], np.arange(n * beams)
    for t in range(steps):
        logits = 2 * torch.randn(n * (beams if t else 1), vocab, generator=g, device="cuda")
        token, parent = dec.select(logits)
        given.append([rows(n * beams, h) for h in (hq, hkv, hkv)])
        o, lse = dec.step(*[x.clone() for x in given[-1]])
        assert int(dec.counts[1]) == 0
        if t % 7 == 3:
            moved, used, end = dec.compact()
            assert end == used
        # attention over every beam's own table, all of it
        ordinary = torch.empty_like(o), torch.empty_like(lse)
        work = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_ATTN, dec.cache, n * beams, width, n * beams, hq), dtype=torch.uint8, device="cuda")
        qr = given[-1][0].clone()
        dec.prompts._rotate(qr, given[-1][1].clone(), dec.prompts._to(np.repeat(np.array(lens) + t, beams)))
        B.fcp_cache_attn(dec.cache, qr, dec._cu, dec.kv_len, dec.pages, dec.scale, *ordinary, work)
        # values are at most 5 or so: each result is off by two bf16 roundings at most, and by a little in 32 bits
        assert float((ordinary[0].float() - o.float()).abs().max()) <= 2.0 ** -6 * 5 and float((ordinary[1] - lse).abs().max()) < 1e-4
    # whom every beam at the end comes from, step by step
    last = np.arange(n * beams)
    order = []
    for t in range(steps - 1, -1, -1):
        order.append(last)
        last = dec.history[t][0].cpu().numpy().reshape(-1)[last] if t else last
    order.reverse()
    alone.prefill(*again, [m for m in lens for _ in range(beams)])
    for t in range(steps):
        alone.step(*[x[torch.from_numpy(order[t]).cuda()].contiguous() for x in given[t]], [1] * (n * beams), weigh=False)
    pages, kv_len = dec.pages.cpu().numpy(), dec.kv_len.cpu().numpy()
    assert kv_len.tolist() == alone.kv_len.tolist()
    for s in range(n * beams):
        for a, b in zip(rows_of(dec.cache, pages[s], kv_len[s], P, fmt), rows_of(alone.cache, alone.pages[s], kv_len[s], P, fmt)):
            assert np.array_equal(a, b), s
    # the tokens of a beam are those on its path, and beams of a prompt differ
    said = dec.sequences()
    for t in range(steps):
        assert np.array_equal(said.reshape(n * beams, steps)[:, t], dec.history[t][1].cpu().numpy().reshape(-1)[order[t]])
    assert all(len({tuple(x) for x in p}) == beams for p in said)
    # a page that several beams hold is there once
    used = {int(p) for s in range(n * beams) for p in pages[s, : -(-int(kv_len[s]) // P)]}
    assert len(used) < sum(-(-int(m) // P) for m in kv_len) and dec.compact()[1] == len(used)


@pytest.mark.gpu
def test_too_few_pages_leave_the_beams_as_they_were():
    import torch
    from paper_2602_21788_amd.decode import BeamDecoder
    rows = lambda n, h: torch.randn(n, h, 64, device="cuda").to(torch.bfloat16)
    dec = BeamDecoder(1, 4, 5, 4, 2, 2, 64, page_tokens=16)
    dec.prefill(rows(20, 2), rows(20, 2), rows(20, 2), [20])
    with pytest.raises(ValueError):
        dec.step(rows(4, 2), rows(4, 2), rows(4, 2))         # nothing chosen
    dec.select(torch.randn(1, 50, device="cuda"))
    dec.step(rows(4, 2), rows(4, 2), rows(4, 2))             # the page that is begun, and three copies of it: the pool is full
    for _ in range(11):
        dec.select(torch.randn(4, 50, device="cuda") - 100 * torch.eye(4, 50, device="cuda"))
        before = dec.pages.clone(), dec.kv_len.clone(), dec.steps
        try:
            dec.step(rows(4, 2), rows(4, 2), rows(4, 2))
        except MemoryError:
            assert torch.equal(dec.pages, before[0]) and torch.equal(dec.kv_len, before[1]) and dec.steps == before[2]
            break
    else:
        raise AssertionError("32 tokens of four beams do not fit 80 slots")
    with pytest.raises(ValueError):
        dec.step(rows(3, 2), rows(3, 2), rows(3, 2))


@pytest.mark.gpu
def test_calls_out_of_turn_and_full_tables_are_refused():
    """Two choices without a step between them; a step where the longest sequence's table is full, which would write over its last token."""
    import torch
    from paper_2602_21788_amd.decode import BeamDecoder
    rows = lambda n, h: torch.randn(n, h, 64, device="cuda").to(torch.bfloat16)
    dec = BeamDecoder(2, 2, 40, 2, 2, 2, 64, page_tokens=16)
    dec.prefill(rows(33, 2), rows(33, 2), rows(33, 2), [30, 3])
    for t in range(3):
        dec.select(torch.randn(4 if t else 2, 50, device="cuda"))
        with pytest.raises(ValueError):
            dec.select(torch.randn(4, 50, device="cuda"))
        if t < 2:
            dec.step(rows(4, 2), rows(4, 2), rows(4, 2))
    codes, pages = dec.cache.k.view(torch.int8).clone(), dec.pages.clone()
    with pytest.raises(MemoryError):
        dec.step(rows(4, 2), rows(4, 2), rows(4, 2))
    assert torch.equal(dec.cache.k.view(torch.int8), codes) and torch.equal(dec.pages, pages) and dec.kv_len.tolist() == [32, 32, 5, 5]


@pytest.mark.gpu
def test_prompts_without_tokens():
    import torch
    from paper_2602_21788_amd.decode import BeamDecoder
    rows = lambda n, h: torch.randn(n, h, 64, device="cuda").to(torch.bfloat16)
    for lens in ([0, 0], [0, 20]):
        dec = BeamDecoder(2, 2, 40, 2, 2, 2, 64, page_tokens=16, rot_dim=0)
        dec.prefill(rows(sum(lens), 2), rows(sum(lens), 2), rows(sum(lens), 2), lens)
        dec.select(torch.randn(2, 50, device="cuda"))
        v = rows(4, 2)
        o, lse = dec.step(rows(4, 2), rows(4, 2), v.clone())
        assert dec.kv_len.tolist() == [m + 1 for m in lens for _ in range(2)]
        # a token alone sees its own value, in e4m3 (half a step of 2^-3), which a bf16 rounding of O follows
        assert float((o[:2].float() - v[:2].float()).abs().max()) <= float(v[:2].abs().max()) * (2.0 ** -4 + 2.0 ** -8)


@pytest.mark.gpu
def test_ended_beams_and_beams_without_candidates():
    """A vocabulary of two tokens, one of which ends a beam: fewer candidates than beams at first, then finished ones stay at their score."""
    import torch
    from paper_2602_21788_amd.decode import BeamDecoder
    rows = lambda n, h: torch.randn(n, h, 64, device="cuda").to(torch.bfloat16)
    dec = BeamDecoder(2, 3, 40, 4, 4, 2, 64, end_token=1, page_tokens=16)
    dec.prefill(rows(30, 4), rows(30, 2), rows(30, 2), [18, 12])
    token, parent = dec.select(torch.zeros(2, 2, device="cuda"))
    assert token.tolist() == [[0, 1, -1]] * 2 and parent.tolist() == [[0, 0, -1], [1, 1, -1]] and dec.done.tolist() == [0, 1, 0] * 2
    o, lse = dec.step(rows(6, 4), rows(6, 2), rows(6, 2))
    assert dec.kv_len.tolist() == [19, 19, 1, 13, 13, 1] and torch.isfinite(lse).all()
    token, parent = dec.select(torch.zeros(6, 2, device="cuda"))
    assert token.tolist() == [[1, 0, 1]] * 2 and parent.tolist() == [[1, 0, 0], [4, 3, 3]] and dec.done.tolist() == [1, 0, 1] * 2
    ln2 = float(np.log(2.0))
    assert np.allclose(dec.score.tolist(), [-ln2, -2 * ln2, -2 * ln2] * 2, rtol=2.0 ** -23)
    dec.step(rows(6, 4), rows(6, 2), rows(6, 2))
    assert dec.kv_len.tolist() == [20] * 3 + [14] * 3
    assert dec.sequences()[0].tolist() == [[1, 1], [0, 0], [0, 1]]


@pytest.mark.gpu
def test_two_steps_in_a_graph():
    """select, fork, append, attention, there and back between two sets of tables, captured once and replayed with new logits and rows; every replay against the same calls made eagerly."""
    import torch
    from paper_2602_21788_amd.decode import CacheDecoder
    g = torch.Generator(device="cuda").manual_seed(9)
    n, beams, hq, hkv, D, P, vocab, m = 3, 4, 8, 2, 128, 32, 3001, 1200          # (tables with which a prompt's beams are worked together)
    rows = n * beams
    draw = lambda r, h: torch.randn(r, h, D, generator=g, device="cuda").to(torch.bfloat16)
    lens = [100, 33, 64]
    q0, k0, v0 = draw(sum(lens), hq), draw(sum(lens), hkv), draw(sum(lens), hkv)
    worlds = []
    for _ in range(2):                                       # one eager, one captured: the same state in tensors of their own
        dec = CacheDecoder(n, 300, m, hq, hkv, D, page_tokens=P, rot_dim=0)
        dec.prefill(q0.clone(), k0.clone(), v0.clone(), lens)
        i32, f32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda"), lambda *s: torch.zeros(*s, device="cuda")
        w = dict(cache=dec.cache, tables=[(i32(rows, m), i32(rows)) for _ in range(2)], score=[f32(n, beams) for _ in range(2)], parent=i32(n, beams), token=i32(n, beams), counts=i32(3),
                 ones=dec._to(np.ones(rows)), cu=dec._to(np.arange(rows + 1)), groups=dec._to(np.arange(n + 1) * beams), shared=dec._to(np.array(lens) // P * P),
                 logits=[f32(rows, vocab) for _ in range(2)], q=[draw(rows, hq) for _ in range(2)], k=[draw(rows, hkv) for _ in range(2)], v=[draw(rows, hkv) for _ in range(2)],
                 o=[torch.empty(rows, hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)], lse=[f32(hq, rows) for _ in range(2)])
        size = lambda b: torch.empty(b, dtype=torch.uint8, device="cuda")
        w["ws"] = [size(B.fcp_beam_scratch_bytes(n, beams, vocab, beams)), size(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_FORK, dec.cache, rows, m)),
                   size(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_SHARED, dec.cache, rows, m, rows, hq))]
        # the first step: the prompts' beams
        B.fcp_cache_fork(dec.cache, dec.pages_d, dec.kv_len_d, dec._to(np.repeat(np.arange(n), beams)), i32(rows), *w["tables"][0], w["counts"], w["ws"][1])
        w["score"][0].copy_(-torch.arange(beams, device="cuda").float().expand(n, beams))
        w["scale"] = dec.scale
        worlds.append(w)

    def two_steps(w):
        for a in range(2):
            B.fcp_beam_select(w["logits"][a], w["score"][a].view(-1), beams, w["parent"], w["token"], w["score"][1 - a], w["ws"][0])
            B.fcp_cache_fork(w["cache"], *w["tables"][a], w["parent"], w["ones"], *w["tables"][1 - a], w["counts"], w["ws"][1])
            pages, kv_len = w["tables"][1 - a]
            B.fcp_cache_append(w["cache"], w["k"][a], w["v"][a], w["cu"], kv_len, pages)
            B.fcp_cache_attn_shared(w["cache"], w["q"][a], w["cu"], kv_len, pages, w["groups"], w["shared"], w["scale"], w["o"][a], w["lse"][a], w["ws"][2])

    eager, captured = worlds
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        two_steps(captured)
    for step in range(5):
        for a in range(2):
            for name, x in (("logits", torch.randn(rows, vocab, generator=g, device="cuda") * 2), ("q", draw(rows, hq)), ("k", draw(rows, hkv)), ("v", draw(rows, hkv))):
                eager[name][a].copy_(x)
                captured[name][a].copy_(x)
        two_steps(eager)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("score", "o", "lse"):
            assert all(torch.equal(x, y) for x, y in zip(eager[name], captured[name])), (step, name)
        for x, y in zip(eager["tables"] + [(eager["parent"], eager["counts"])], captured["tables"] + [(captured["parent"], captured["counts"])]):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]), step
        assert int(captured["counts"][1]) == 0 and captured["tables"][0][1].tolist() == [x + 2 * step + 2 for x in lens for _ in range(beams)]


@pytest.mark.gpu
def test_small_run():
    """python -m paper_2602_21788_amd.decode runs."""
    from paper_2602_21788_amd import decode
    decode.main()
