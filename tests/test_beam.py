"""Beam selection against the definition in 64 bits (numpy), and its refusals (on the CPU)."""
import numpy as np
import pytest

from paper_2602_21788_amd import binding as B

BIG = float(np.finfo(np.float32).max)


# ---- the definition -------------------------------------------------------------------------------------------------------------------------
def select(x, score, beams, keep, done=None, end=-1):
    """x [rows, vocab], score [rows] float64.  Returns parent, token, score (float64), done, [n_prompts, keep]."""
    rows = len(x)
    x = np.minimum(np.where(np.isnan(x), -np.inf, x.astype(np.float64)), BIG)
    out = []
    for p in range(rows // beams):
        found = []
        for r in range(p * beams, (p + 1) * beams):
            if not score[r] > -np.inf:
                continue
            if done is not None and done[r]:
                found.append((-float(score[r]), r, end, 1))
                continue
            v = x[r]
            top = v.max()
            if top == -np.inf:
                continue
            lse = top + np.log(np.exp(v - top).sum())
            best = np.argsort(-v, kind="stable")[:keep]
            found += [(-(float(score[r]) + float(v[t] - lse)), r, int(t), int(t == end)) for t in best if v[t] > -np.inf]
        found.sort()
        # the kernels' logarithm is off by 5.4e-11 at most: what the oracle's 64 bits call different must lie further apart than twice that, or the case says nothing
        gaps = np.diff([f[0] for f in found[: keep + 1] if np.isfinite(f[0])])
        assert ((gaps == 0) | (gaps > 1e-9)).all(), "the inputs have candidates too close to each other"
        found = found[:keep] + [(np.inf, -1, -1, 0)] * (keep - len(found))
        out.append(found)
    a = np.array([[(f[1], f[2], f[3]) for f in q] for q in out], np.int64).reshape(-1, keep, 3)
    return a[..., 0], a[..., 1], -np.array([[f[0] for f in q] for q in out]).reshape(-1, keep), a[..., 2]


def test_definition():
    """Uniform logits: every token costs ln vocab; a beam that is done costs nothing; the first beams and tokens win ties."""
    parent, token, score, over = select(np.zeros((4, 8)), np.array([0.0, -0.5, -np.inf, -3.0]), 2, 3, np.array([0, 1, 0, 0]), 7)
    assert parent.tolist() == [[1, 0, 0], [3, 3, 3]] and token.tolist() == [[7, 0, 1], [0, 1, 2]] and over.tolist() == [[1, 0, 0], [0, 0, 0]]
    assert np.allclose(score, [[-0.5, -np.log(8), -np.log(8)], [-3 - np.log(8)] * 3], atol=1e-15)
    parent, token, score, over = select(np.array([[1.0, -np.inf, np.nan]]), np.array([0.0]), 1, 2)
    assert parent.tolist() == [[0, -1]] and token.tolist() == [[0, -1]] and score.tolist() == [[0.0, -np.inf]]


# ---- CPU ------------------------------------------------------------------------------------------------------------------------------------
def _call(**kw):
    """A call with addresses that nobody looks at: every one below fails first, or has nothing to do."""
    f = 0x10000
    a = lambda name, v: kw.get(name, v)
    return B.lib().fcp_beam_select(a("logits", f), a("type", 0), a("row", 100), a("n_prompts", 2), a("beams", 3), a("vocab", 100), a("score", f), a("done", f), a("end", 5),
                                   a("keep", 6), a("parent", f), a("token", f), a("new_score", f + 4), a("new_done", f + 64), a("scratch", f), a("bytes", 1 << 40), None)


def test_refusals_come_before_any_device_work():
    bad, no, full = B.FCP_ERR_INVALID_ARG, B.FCP_ERR_UNSUPPORTED, B.FCP_ERR_CAPACITY
    for kw in (dict(n_prompts=-1), dict(beams=0), dict(vocab=0), dict(keep=0), dict(end=-2), dict(end=100), dict(logits=None), dict(score=None), dict(parent=None),
               dict(token=None), dict(new_score=None), dict(row=99), dict(logits=0x10001), dict(type=1, logits=0x10002), dict(score=0x10002), dict(parent=0x10001),
               dict(token=0x10002), dict(new_score=0x10001), dict(new_score=0x10000), dict(new_done=0x10000), dict(scratch=None), dict(scratch=0x10010)):
        assert _call(**kw) == bad, kw
        assert b"fcp_beam_select" in B.lib().fcp_last_error()
    for kw in (dict(type=2), dict(beams=257), dict(keep=65), dict(vocab=(1 << 30) + 1, row=1 << 31), dict(n_prompts=1 << 22, beams=4), dict(n_prompts=1 << 30, beams=4),
               dict(n_prompts=1 << 13, beams=256, vocab=1 << 16, row=1 << 16)):
        assert _call(**kw) == no, kw
    need = B.fcp_beam_scratch_bytes(2, 3, 100, 6)
    assert _call(bytes=need - 1) == full
    assert _call(n_prompts=0, logits=None) == B.FCP_OK
    for args in ((-1, 3, 100, 6), (2, 0, 100, 6), (2, 3, 0, 6), (2, 3, 100, 0), (2, 257, 100, 6), (2, 3, 100, 65), (1 << 22, 4, 100, 6)):
        with pytest.raises(B.FcpError):
            B.fcp_beam_scratch_bytes(*args)
    assert B.fcp_beam_scratch_bytes(0, 3, 100, 6) > 0


def test_scratch_grows_with_the_call():
    sizes = [B.fcp_beam_scratch_bytes(n, b, v, k) for n, b, v, k in ((1, 1, 1, 1), (1, 4, 32000, 8), (8, 5, 50001, 10), (64, 8, 131072, 16), (64, 8, 131072, 64))]
    assert sizes == sorted(sizes) and sizes[0] >= 256


# ---- GPU ------------------------------------------------------------------------------------------------------------------------------------
def _run(x, score, beams, keep, done=None, end=-1, pad=0, dtype="f32", stream=None):
    """Device results as numpy, from logits that lie in a larger tensor full of large values."""
    import torch
    rows, vocab = x.shape
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    whole = torch.full((rows * (vocab + pad) + 16,), 1e9, dtype=t, device="cuda")
    logits = whole[: rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    logits.copy_(torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda())
    n = rows // beams
    out = [torch.full((n + 1, keep), v, dtype=d, device="cuda") for v, d in ((77, torch.int32), (77, torch.int32), (7.5, torch.float32), (9, torch.uint8))]
    scratch = torch.full((B.fcp_beam_scratch_bytes(n, beams, vocab, keep),), 255, dtype=torch.uint8, device="cuda")
    B.fcp_beam_select(logits, torch.from_numpy(np.asarray(score, np.float32)).cuda(), beams, out[0][:n], out[1][:n], out[2][:n], scratch,
                      None if done is None else torch.from_numpy(np.asarray(done, np.uint8)).cuda(), end, out[3][:n], stream)
    torch.cuda.synchronize()
    for o, v in zip(out, (77, 77, 7.5, 9)):
        assert (o[n] == v).all()                             # nothing behind the last prompt
    return [o[:n].cpu().numpy() for o in out]


def _check(x, score, beams, keep, done=None, end=-1, **kw):
    import torch
    if kw.get("dtype") == "bf16":
        x = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).float().numpy()
    x, score = np.asarray(x, np.float32), np.asarray(score, np.float32)
    want = select(x, score.astype(np.float64), beams, keep, done, end)
    got = _run(x, score, beams, keep, done, end, **kw)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]) and np.array_equal(got[3], want[3])
    there = np.isfinite(want[2])
    assert np.array_equal(got[2][~there], want[2][~there])
    # one rounding to 32 bits, and the logarithm
    assert (np.abs(got[2][there] - want[2][there]) <= 2.0 ** -24 * np.abs(want[2][there]) + 1e-10).all()


def _scores(rng, rows):
    return (-rng.random(rows) * 20).astype(np.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prompts, beams, vocab, keep, pad", [
    (1, 1, 1, 1, 0), (1, 1, 5, 3, 0), (2, 3, 63, 6, 1), (3, 2, 64, 4, 0), (1, 4, 255, 8, 3), (2, 2, 2047, 4, 0), (2, 2, 2048, 4, 0), (2, 2, 2049, 4, 0), (5, 7, 4999, 14, 0),
    (1, 4, 32000, 8, 0), (1, 5, 50001, 64, 7), (1, 1, 100, 64, 0), (1, 256, 40, 64, 0), (70, 8, 300, 16, 0), (64, 8, 8193, 9, 5), (128, 4, 8192, 1, 0), (30, 2, 70001, 5, 0)])
def test_sizes(dtype, prompts, beams, vocab, keep, pad):
    rng = np.random.default_rng(vocab + keep)
    x = rng.standard_normal((prompts * beams, vocab)) * 2.5
    _check(x, _scores(rng, prompts * beams), beams, keep, dtype=dtype, pad=pad)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prompts, beams, vocab, keep, pad", [(260, 4, 16385, 5, 3), (128, 8, 17000, 64, 0), (40, 8, 70001, 33, 1), (1030, 1, 5001, 1, 0)])
def test_many_rows_of_long_chunks(dtype, prompts, beams, vocab, keep, pad):
    rng = np.random.default_rng(vocab + keep)
    x = rng.standard_normal((prompts * beams, vocab)) * 2.5
    _check(x, _scores(rng, prompts * beams), beams, keep, dtype=dtype, pad=pad)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [6, 600])                     # chunks of 2048, of 8192
@pytest.mark.parametrize("first, last, keep", [(0, 1000, 64), (4000, 5500, 30), (8191, 8193, 3), (16000, 16700, 10), (100, 164, 64), (2047, 9000, 64)])
def test_masks_that_leave_a_run_of_tokens(rows, dtype, first, last, keep):
    """Few of a block's threads hold anything, or as few groups as are kept: more logits than a block lists may be among the best.  Beams of different masks beside each other, values that repeat."""
    rng = np.random.default_rng(first + keep)
    x = np.full((rows, 16700), -np.inf)
    x[:, first:last] = np.round(rng.standard_normal((rows, last - first)) * 4, 1)
    x[1] = np.where(rng.random(16700) < 0.01, x[1], -np.inf)
    x[2, first:last] = 1.5
    x[3, first:last] = np.where(np.arange(first, last) % 3 == 0, -7.0, -np.inf)
    _check(x, _scores(rng, rows), 2, keep, dtype=dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [7, 700])                     # chunks of 2048, of 8192
@pytest.mark.parametrize("spread", [0.0, 1e-3, 5.0, 200.0, 900.0])
def test_logarithm_of_the_sum(rows, spread):
    """The beam's score takes away nearly all of the best token's -ln(probability), so that its rounding to 32 bits says nothing and what the logarithm is off by shows: 5.4e-11 in a chunk's sum and 4.3e-11 in
    the factor that brings it to another chunk's greatest logit at most, and a few roundings of 64 bits of lse itself.  Greatest logits on both sides of 1024, where the sums change their way."""
    rng = np.random.default_rng(int(spread))
    top = np.resize([0.0, 1.0, -3.3, 88.7, -1023.9, 1023.99, 1024.0, 1024.5, -1025.0, 30000.0, -70000.0], rows)
    x = (top[:, None] - spread * rng.random((rows, 9001))).astype(np.float32)
    v = x.astype(np.longdouble)
    most = v.max(1)
    lse = most + np.log(np.exp(v - most[:, None]).sum(1))
    score = (lse - most).astype(np.float32)
    want = score.astype(np.longdouble) - (lse - most)
    got = _run(x, score, 1, 1)[2][:, 0]
    assert (np.abs(got - want) <= 1e-10 + 2.0 ** -24 * np.abs(want) + 2.0 ** -51 * np.abs(lse)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [6, 600])                     # chunks of 2048, of 8192
@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two", "steps", "one_high", "zeros"])
def test_orders(rows, kind):
    """Logits in an order that fills a block's list: equal ones (the lowest tokens win), rising ones (the list is as long as it can be), few different values."""
    vocab, keep = 9000, 33
    x = {"equal": np.full(vocab, 3.5), "rising": np.arange(vocab) / 8, "falling": -np.arange(vocab) / 8, "two": (np.arange(vocab) % 7 == 3) * 2.0,
         "steps": np.arange(vocab) // 64 / 4.0, "one_high": np.where(np.arange(vocab) == 8999, 9.0, np.sin(np.arange(vocab))),
         "zeros": np.where(np.arange(vocab) % 2 == 0, -0.0, 0.0)}[kind]
    x = np.broadcast_to(x, (rows, vocab))
    # beams with the same logits: scores a step apart, or equal (the lower beam first)
    score = np.where(np.arange(rows) % 3 == 2, -1.0, -1.0 - 1e-3 * (np.arange(rows) % 3))
    _check(x, score, 3, keep)
    _check(x, np.zeros(rows), 3, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [12, 1200])
def test_masks_and_values_that_are_not_finite(rows, dtype):
    rng = np.random.default_rng(2)
    vocab, beams, keep = 3000, 4, 8
    x = rng.standard_normal((rows, vocab)) * 3
    x[0] = -np.inf                                           # a row that offers nothing
    x[1, :] = np.nan
    x[2, 5:] = -np.inf                                       # fewer candidates than are kept
    x[4:8] = -np.inf                                         # a prompt that offers nothing ..
    x[5, 17] = 1.0                                           # .. but one token
    x[8, 100:200] = np.nan
    x[9, 50] = np.inf
    x[9, 60] = np.inf
    x[10, 70] = 1e38
    score = _scores(rng, rows)
    score[3], score[11] = -np.inf, np.nan
    done = np.zeros(rows, np.uint8)
    done[[7, 10]] = 1, 255
    for end in (-1, 2):
        _check(x, score, beams, keep, done, end, dtype=dtype)
    _check(x, score, beams, keep, None, 2, dtype=dtype)
    _check(x, np.full(rows, -np.inf), beams, keep, dtype=dtype)
    _check(x, np.where(np.arange(rows) % beams == 0, 0.0, -np.inf), beams, keep, dtype=dtype)      # a first step: one beam of each prompt


@pytest.mark.gpu
def test_signalling_nans_are_masks_too():
    import torch
    bits = torch.full((2, 100), 0x3f80, dtype=torch.int16)
    bits[0, ::3], bits[1, ::2] = 0x7f81, -0x7f                # 0x7f81, 0xff81
    bits[:, 50] = 0x4000
    out = [torch.empty(2, 3, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    scratch = torch.empty(B.fcp_beam_scratch_bytes(2, 1, 100, 3), dtype=torch.uint8, device="cuda")
    B.fcp_beam_select(bits.cuda().view(torch.bfloat16), torch.zeros(2, device="cuda"), 1, *out, scratch)
    assert out[1].tolist() == [[50, 1, 2], [50, 1, 3]]
    assert torch.isfinite(out[2]).all()


@pytest.mark.gpu
def test_great_logits():
    """Sums keep their meaning where exp(x) has no value: the scores are those of x - greatest."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((8, 2500)) * 3
    for shift in (-1e4, 300.0, 3e6):
        _check((x + shift).astype(np.float32), _scores(rng, 8), 2, 5)


@pytest.mark.gpu
def test_graph_replays_follow_their_inputs_beside_another_stream():
    """Two graphs with work space of their own, replayed with new logits, other work on another stream between them."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    V, beams, keep, n = 7001, 4, 8, 3
    mk = lambda: (torch.randn(n * beams, V, generator=g, device="cuda").to(torch.bfloat16), -5 * torch.rand(n * beams, generator=g, device="cuda"))
    outs = lambda: [torch.empty(n, keep, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    space = lambda: torch.empty(B.fcp_beam_scratch_bytes(n, beams, V, keep), dtype=torch.uint8, device="cuda")
    graphs = []
    for _ in range(2):
        x, s = mk()
        o, w, graph = outs(), space(), torch.cuda.CUDAGraph()
        B.fcp_beam_select(x, s, beams, *o, w)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            B.fcp_beam_select(x, s, beams, *o, w)
        graphs.append((x, s, o, graph, w))
    other = torch.cuda.Stream()
    for _ in range(4):
        eager = []
        for x, s, o, graph, _ in graphs:
            nx, ns = mk()
            x.copy_(nx)
            s.copy_(ns)
            graph.replay()
        with torch.cuda.stream(other):
            other.wait_stream(torch.cuda.default_stream())
            for x, s, *_ in graphs:
                e = outs()
                B.fcp_beam_select(x, s, beams, *e, space())
                eager.append(e)
        torch.cuda.synchronize()
        for e, (_, _, o, _, _) in zip(eager, graphs):
            assert all(torch.equal(a, b) for a, b in zip(e, o))


@pytest.mark.gpu
def test_binding_refuses_tensors_of_other_types_and_sizes():
    import torch
    x, s = torch.zeros(4, 50, device="cuda"), torch.zeros(4, device="cuda")
    out = lambda: [torch.empty(2, 3, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    w = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    B.fcp_beam_select(x, s, 2, *out(), w)
    for bad in (lambda o: B.fcp_beam_select(x.half(), s, 2, *o, w), lambda o: B.fcp_beam_select(x.T.contiguous().T, s, 2, *o, w), lambda o: B.fcp_beam_select(x, s, 3, *o, w),
                lambda o: B.fcp_beam_select(x, s[:3], 2, *o, w), lambda o: B.fcp_beam_select(x, s.double(), 2, *o, w), lambda o: B.fcp_beam_select(x, s, 2, o[0].long(), o[1], o[2], w),
                lambda o: B.fcp_beam_select(x, s, 2, o[0], o[1][:, :2], o[2], w), lambda o: B.fcp_beam_select(x, s, 2, o[0], o[1], o[2].double(), w),
                lambda o: B.fcp_beam_select(x, s, 2, *o, w, done=torch.zeros(4, device="cuda")), lambda o: B.fcp_beam_select(x, s, 2, *o, w, done=torch.zeros(3, dtype=torch.uint8, device="cuda")),
                lambda o: B.fcp_beam_select(x.cpu(), s, 2, *o, w)):
        with pytest.raises(ValueError):
            bad(out())
