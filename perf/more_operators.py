"""Performance cases of the operators that answer with several continuations of a prompt over the paged 8-bit cache:

  beam     the best (beam, token) candidates of every prompt, from the beams' logits and the scores so far
  fork     the sequences of the next step out of those of this one: tables that share what is read only, copies of the pages
           that several would write, fresh pages for the new tokens
  compact  pages in use moved to the lowest numbers of the pool
  shared   attention of new tokens over the cache where the sequences of a group have a common beginning

Where `own` is false, run() computes the plain forms in elementary torch operations; where it is true, it calls the package.
Lengths, and who continues whom, follow from the case, values from the seed.  Ragged lengths: i has longest / 20^frac(0.618 i).
"""
import math

import numpy as np
import torch

own = False

#: (query heads, KV heads)
HEADS = [(4, 4), (8, 8), (6, 2), (10, 2), (8, 1), (32, 8), (40, 8)]
MOST_KEEP = 64


def listed():
    return [
        # the smallest selection: four beams of one prompt
        {"name": "beam_4_of_32k", "op": "beam", "prompts": 1, "beams": 4, "vocab": 32000, "pad": 0, "type": "bf16", "keep": 8, "masked": 0.0,
         "done": False},
        # an odd vocabulary in fp32, rows next to each other (so that most begin off 16 bytes), some beams at their end
        {"name": "beam_8x5_of_50001_f32", "op": "beam", "prompts": 8, "beams": 5, "vocab": 50001, "pad": 0, "type": "f32", "keep": 10,
         "masked": 0.0, "done": True},
        # a large batch over a large vocabulary, half of it ruled out by a grammar
        {"name": "beam_64x8_of_131k", "op": "beam", "prompts": 64, "beams": 8, "vocab": 131072, "pad": 0, "type": "bf16", "keep": 16,
         "masked": 0.5, "done": True},
        # a step of eight beams of one prompt
        {"name": "fork_8", "op": "fork", "prompts": 1, "beams": 8, "longest": 1000, "own": 37, "new": 1, "hkv": 4, "head_dim": 64, "page": 16,
         "format": "e4m3"},
        # a step of a serving batch
        {"name": "fork_256", "op": "fork", "prompts": 32, "beams": 8, "longest": 8001, "own": 100, "new": 1, "hkv": 8, "head_dim": 128,
         "page": 64, "format": "int8"},
        # prompts whose beams begin: every prompt's last page is copied for all of its beams but one
        {"name": "fork_start_1024", "op": "fork", "prompts": 64, "beams": 16, "longest": 16383, "own": 0, "new": 1, "hkv": 8, "head_dim": 128,
         "page": 64, "format": "e4m3"},
        # a small pool after some sequences ended
        {"name": "compact_8", "op": "compact", "seqs": 8, "longest": 600, "fill": 0.7, "hkv": 4, "head_dim": 64, "page": 16, "format": "int8"},
        # a large one, a bit more than half in use
        {"name": "compact_64_long", "op": "compact", "seqs": 64, "longest": 16384, "fill": 0.55, "hkv": 8, "head_dim": 128, "page": 64,
         "format": "e4m3"},
        # four beams of a short prompt, a small model with narrow heads
        {"name": "shared_4_of_500", "op": "shared", "groups": 1, "seqs": 4, "longest": 500, "own": 20, "new": 1, "hq": 4, "hkv": 4,
         "head_dim": 64, "page": 16, "format": "e4m3"},
        # sixty-four samples of one long prompt
        {"name": "shared_64_of_16k", "op": "shared", "groups": 1, "seqs": 64, "longest": 16384, "own": 300, "new": 1, "hq": 32, "hkv": 8,
         "head_dim": 128, "page": 64, "format": "e4m3"},
        # a serving batch: eight beams of each of sixteen ragged prompts
        {"name": "shared_16x8_ragged", "op": "shared", "groups": 16, "seqs": 8, "longest": 8000, "own": 200, "new": 1, "hq": 32, "hkv": 8,
         "head_dim": 128, "page": 32, "format": "int8"},
        # eight questions of 256 tokens about one document
        {"name": "shared_8_chunks_of_256", "op": "shared", "groups": 1, "seqs": 8, "longest": 4001, "own": 0, "new": 256, "hq": 40, "hkv": 8,
         "head_dim": 128, "page": 64, "format": "e4m3"},
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the ranges the listed ones stand for, no dearer than the dearest of them of its operator."""
    while True:
        op = rng.choice(["beam", "beam", "beam", "fork", "fork", "compact", "shared", "shared", "shared"])
        case = {"op": op}
        if op == "beam":
            beams = _log_between(rng, 1, 16)
            vocab = _log_between(rng, 100, 131072)
            case.update(prompts=_log_between(rng, 1, 64), beams=beams, vocab=vocab, pad=rng.choice([0, 0, -vocab % 64]), type=rng.choice(["bf16", "bf16", "f32"]),
                        keep=rng.randint(beams, min(2 * beams, MOST_KEEP)), masked=rng.choice([0.0, 0.0, 0.5, 0.9]), done=rng.random() < 0.5)
        else:
            hq, hkv = rng.choice(HEADS)
            case.update(hkv=hkv, head_dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 64, 128]), format=rng.choice(["e4m3", "int8"]))
            if op == "fork":
                case.update(prompts=_log_between(rng, 1, 64), beams=_log_between(rng, 1, 16), longest=_log_between(rng, 1, 16384),
                            own=rng.choice([0, _log_between(rng, 1, 300)]), new=rng.choice([1, 1, 1, 0, _log_between(rng, 2, 300)]))
            elif op == "compact":
                case.update(seqs=_log_between(rng, 1, 64), longest=_log_between(rng, 20, 16384), fill=rng.uniform(0.3, 0.95))
            else:
                case.update(hq=hq, groups=_log_between(rng, 1, 16), seqs=_log_between(rng, 1, 64), longest=_log_between(rng, 1, 16384),
                            own=rng.choice([0, _log_between(rng, 1, 300)]), new=rng.choice([1, 1, 1, _log_between(rng, 2, 256)]))
        most = [work(c) for c in listed() if c["op"] == op]
        mine = work(case)
        if mine["bytes"] <= max(w["bytes"] for w in most) and mine["flops"] <= max(w["flops"] for w in most) and _padded(case) <= 1 << 31:
            return case


# ---- layouts ------------------------------------------------------------------------------------------------------------
def _ragged(n, longest, least=1, offset=0):
    return [max(least, int(longest / 20 ** ((0.618 * (i + offset)) % 1))) for i in range(n)]


def _prompts(case):
    """Lengths of the prompts."""
    return _ragged({"fork": case.get("prompts"), "shared": case.get("groups"), "compact": case.get("seqs")}[case["op"]], case["longest"])


def _parents(case):
    """fork: who the sequences of the next step continue.  The better beams have more continuations."""
    beams = case["beams"]
    if case["own"] == 0:
        return [p for p in range(case["prompts"]) for _ in range(beams)]
    return [p * beams + int(beams * ((0.618 * (p * beams + b) + 0.3) % 1) ** 2) for p in range(case["prompts"]) for b in range(beams)]


def _old_lens(case):
    """fork: cached tokens of the sequences of this step."""
    if case["own"] == 0:
        return _prompts(case)
    return [n + case["own"] for n in _prompts(case) for _ in range(case["beams"])]


def _own_lens(case):
    """shared: tokens of every sequence behind its prompt, new ones included."""
    n = case["groups"] * case["seqs"]
    return [o + case["new"] for o in (_ragged(n, case["own"], 0, 1) if case["own"] else [0] * n)]


def _padded(case):
    """Elements of a rectangle that holds all keys, or all scores, or the logits: what the plain form needs at once."""
    if case["op"] == "beam":
        return case["prompts"] * case["beams"] * case["vocab"]
    if case["op"] != "shared":
        return 0
    L, n = case["longest"] + max(_own_lens(case)), case["groups"] * case["seqs"]
    return n * max(L * case["hkv"] * case["head_dim"], case["hq"] * case["new"] * L)


def _token_bytes(case):
    """Keys, values and weight of a cached token."""
    return case["hkv"] * (2 * case["head_dim"] + 4)


def work(case):
    """What the operator cannot do without: inputs read once, outputs written once, and the products."""
    if case["op"] == "beam":
        n = case["prompts"] * case["beams"] * case["vocab"]
        # (beams at their end are not read: one in eight)
        live = 7 / 8 if case["done"] and case["beams"] > 1 else 1
        return {"bytes": int(n * live) * (2 if case["type"] == "bf16" else 4) + 16 * case["prompts"] * (case["beams"] + case["keep"]), "flops": 4 * n}
    D, hkv, P = case["head_dim"], case["hkv"], case["page"]
    if case["op"] == "compact":
        used = sum(-(-n // P) for n in _prompts(case))
        # pages lie anywhere, so what is past the first `used` numbers moves
        moved = int(used * (1 - case["fill"]))
        return {"bytes": 2 * moved * (P * _token_bytes(case) + 8 * hkv) + 8 * used, "flops": 0}
    if case["op"] == "fork":
        lens, parents = _old_lens(case), _parents(case)
        copied = pages = 0
        for s, p in enumerate(parents):
            pages += -(-(lens[p] + case["new"]) // P)
            if case["new"] and lens[p] % P and p in parents[:s]:
                n = lens[p] % P
                copied += hkv * (D * (n + -(-n // 16) * 16) + 4 * n + 8)
        return {"bytes": 2 * copied + 4 * (pages + sum(-(-n // P) for n in lens)), "flops": 0}
    group, own_lens = case["seqs"], _own_lens(case)
    keys, pairs = sum(_prompts(case)) + sum(own_lens), 0
    for i, o in enumerate(own_lens):
        L, n = _prompts(case)[i // group] + o, case["new"]
        pairs += n * (2 * L - n + 1) // 2
    rows = case["new"] * len(own_lens) * case["hq"]
    return {"bytes": keys * hkv * 2 * D + rows * (4 * D + 4) + 8 * hkv * (keys // P), "flops": 4 * pairs * D * case["hq"]}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _int(values):
    return torch.from_numpy(np.ascontiguousarray(values, dtype=np.int32)).cuda()


def _v_pages(v):
    """Value rows [..., page, D] in the cache's order [..., page / 16, D, 16]."""
    *lead, P, D = v.shape
    return v.reshape(*lead, P // 16, 16, D).transpose(-1, -2)


def _v_rows(v):
    """The reverse of _v_pages."""
    *lead, n, D, _ = v.shape
    return v.transpose(-1, -2).reshape(*lead, n * 16, D)


def _pool(gen, case, n_pages):
    """A cache of n_pages pages whose every slot holds a token."""
    shape = (n_pages, case["hkv"], case["page"], case["head_dim"])
    pool = {}
    for name in ("k", "v"):
        x = _normal(gen, *shape)
        x[..., :: 32] *= 3
        # a power of two whose format's largest value is beyond the page's largest magnitude
        e = torch.frexp(x.abs().amax((2, 3)))[1] - (8 if case["format"] == "e4m3" else 6)
        x = torch.ldexp(x, -e[:, :, None, None])
        codes = x.to(torch.float8_e4m3fn) if case["format"] == "e4m3" else x.round().clamp(-127, 127).to(torch.int8)
        pool[name] = (codes if name == "k" else _v_pages(codes)).contiguous()
        pool[name + "_scale"] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
        del x, codes
    pool["weight"] = (torch.exp(2 * _normal(gen, *shape[:3])) * 64).floor() / 64
    return pool


def _fill(counts, numbers):
    """Tables of the given numbers of pages, taken from `numbers` in order; -1 behind them."""
    table = np.full((len(counts), max(max(counts), 1)), -1, np.int32)
    at = np.concatenate([[0], np.cumsum(counts)])
    for i, c in enumerate(counts):
        table[i, :c] = numbers[at[i]: at[i + 1]]
    return table


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 32))
    return globals()["_prepare_" + case["op"]](case, gen, rs)


def _prepare_beam(case, gen, rs):
    rows, V, keep = case["prompts"] * case["beams"], case["vocab"], case["keep"]
    x = torch.empty(rows, V + case["pad"], dtype=torch.bfloat16 if case["type"] == "bf16" else torch.float32, device="cuda")
    for r in range(0, rows, 64):                                         # (a few rows at a time: the rectangle in 32 bits is large)
        part = 2.5 * _normal(gen, *x[r: r + 64].shape)
        if case["masked"]:
            part.masked_fill_(torch.rand(part.shape, generator=gen, device="cuda") < case["masked"], -math.inf)
        x[r: r + 64] = part
    # cumulative log-probabilities, the best beam first
    score = -torch.cumsum(torch.rand(case["prompts"], case["beams"], generator=gen, device="cuda"), 1) * 3 - 5
    done = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    if case["done"] and case["beams"] > 1:
        done[torch.from_numpy(rs.permutation(rows)[: rows // 8]).cuda()] = 1
    s = {"case": case, "logits": x[:, :V], "score": score.reshape(-1).contiguous(), "done": done, "end": 2}
    for name, t in (("parent", torch.int32), ("token", torch.int32), ("new_score", torch.float32), ("new_done", torch.uint8)):
        s[name] = torch.empty(case["prompts"], keep, dtype=t, device="cuda")
    return s


def _prepare_fork(case, gen, rs):
    P, beams, prompts = case["page"], case["beams"], _prompts(case)
    lens, parents, new = _old_lens(case), _parents(case), case["new"]
    own_step = case["own"] > 0
    width = -(-(max(lens) + new) // P) + 1
    common = [n // P if own_step else -(-n // P) for n in prompts]       # pages of a prompt that its sequences share
    private = [-(-n // P) - common[i // beams] for i, n in enumerate(lens)] if own_step else []
    fresh = sum(-(-(lens[p] + new) // P) - -(-lens[p] // P) + 1 for p in parents)
    used = sum(common) + sum(private)
    n_pages = used + fresh + used // 8 + 16
    numbers = rs.permutation(n_pages)                                    # pages of a cache in use lie anywhere
    pages = np.full((len(lens), width), -1, np.int32)
    a, b = _fill(common, numbers), _fill(private, numbers[sum(common):]) if own_step else None
    for i in range(len(lens)):
        p = i // beams if own_step else i
        pages[i, : common[p]] = a[p, : common[p]]
        if own_step:
            pages[i, common[p]: common[p] + private[i]] = b[i, : private[i]]
    busy = np.zeros(n_pages, np.uint8)
    busy[numbers[used: used + used // 16]] = 1                           # held by sequences that are not in the batch
    s = {"case": case, "kv_len": _int(lens), "pages": _int(pages), "parent": _int(parents), "news": _int([new] * len(parents)),
         "busy": torch.from_numpy(busy).cuda(), "new_pages": _int(np.zeros((len(parents), width))), "new_len": _int([0] * len(parents)),
         "counts": _int([0] * 3)}
    s.update(_pool(gen, case, n_pages))
    return s


def _prepare_compact(case, gen, rs):
    P, lens = case["page"], _prompts(case)
    counts = [-(-n // P) for n in lens]
    n_pages = max(int(sum(counts) / case["fill"]), sum(counts) + 1)
    numbers = rs.permutation(n_pages)
    pages = _fill(counts, numbers)
    busy = np.zeros(n_pages, np.uint8)
    busy[numbers[-1]] = 1
    s = {"case": case, "kv_len": _int(lens), "pages": _int(pages), "busy": torch.from_numpy(busy).cuda(), "new_pages": _int(np.zeros(pages.shape)),
         "counts": _int([0] * 3)}
    s.update(_pool(gen, case, n_pages))
    return s


def _prepare_shared(case, gen, rs):
    P, D, hq, group, own_lens = case["page"], case["head_dim"], case["hq"], case["seqs"], _own_lens(case)
    prompts = _prompts(case)
    n = len(own_lens)
    lens = [prompts[i // group] + o for i, o in enumerate(own_lens)]
    common = [m // P for m in prompts]                                   # (as forking leaves them: a prompt's last page is every sequence's own)
    private = [-(-m // P) - common[i // group] for i, m in enumerate(lens)]
    numbers = rs.permutation(sum(common) + sum(private))
    a, b = _fill(common, numbers), _fill(private, numbers[sum(common):])
    pages = np.full((n, -(-max(lens) // P)), -1, np.int32)
    for i in range(n):
        c = common[i // group]
        pages[i, :c] = a[i // group, :c]
        pages[i, c: c + private[i]] = b[i, : private[i]]
    tq = n * case["new"]
    q = _normal(gen, tq, hq, D)
    q[:, :, :: 32] *= 3
    s = {"case": case, "kv_len": _int(lens), "pages": _int(pages), "cu": _int(np.arange(n + 1) * case["new"]),
         "groups": _int(np.arange(case["groups"] + 1) * group), "shared": _int([c * P for c in common]), "scale": 1 / math.sqrt(D),
         "q": q.to(torch.bfloat16), "o": torch.empty(tq, hq, D, dtype=torch.bfloat16, device="cuda"),
         "lse": torch.empty(hq, tq, dtype=torch.float32, device="cuda")}
    s.update(_pool(gen, case, len(numbers)))
    return s


# ---- the operators ------------------------------------------------------------------------------------------------------
def _cache(s):
    """The package, its view of the cache in `s`, and work space of the size it asks for: made once."""
    import paper_2602_21788_amd as fcp
    if "cache" not in s:
        c = s["case"]
        s["cache"] = fcp.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["weight"])
        which = {"fork": fcp.FCP_SCRATCH_CACHE_FORK, "compact": fcp.FCP_SCRATCH_CACHE_COMPACT, "shared": fcp.FCP_SCRATCH_CACHE_SHARED}[c["op"]]
        n = fcp.fcp_cache_scratch_bytes(which, s["cache"], (s["new_pages"] if "new_pages" in s else s["pages"]).shape[0], s["pages"].shape[1],
                                        s["q"].shape[0] if "q" in s else 0, c.get("hq", c["hkv"]))
        s["scratch"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return fcp, s["cache"]


def run(s):
    return globals()["_run_" + s["case"]["op"]](s)


def _run_beam(s):
    case = s["case"]
    if own:
        import paper_2602_21788_amd as fcp
        if "scratch" not in s:
            n = fcp.fcp_beam_scratch_bytes(case["prompts"], case["beams"], case["vocab"], case["keep"])
            s["scratch"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        fcp.fcp_beam_select(s["logits"], s["score"], case["beams"], s["parent"], s["token"], s["new_score"], s["scratch"], done=s["done"],
                            end_token=s["end"], new_done=s["new_done"])
    else:
        # in 64 bits, since candidates of different beams may lie next to each other
        B, n, V, keep, end = case["beams"], case["prompts"], case["vocab"], case["keep"], s["end"]
        x = s["logits"].double()
        top = x.amax(1, keepdim=True).clamp(min=-1e300)
        x.sub_(top)
        x.sub_(torch.log(torch.exp(x).sum(1, keepdim=True)).clamp(min=-1e300))
        x.add_(s["score"].double()[:, None])
        over = s["done"].bool()[:, None]
        x.masked_fill_(over, -math.inf)
        x[:, end] = torch.where(over[:, 0], s["score"].double(), x[:, end])
        best, at = x.reshape(n, B * V).sort(dim=1, descending=True, stable=True)
        best, at = best[:, :keep], at[:, :keep]
        if keep > B * V:
            best, at = torch.nn.functional.pad(best, (0, keep - B * V), value=-math.inf), torch.nn.functional.pad(at, (0, keep - B * V))
        there = best > -math.inf
        parent = torch.where(there, at // V + B * torch.arange(n, device="cuda")[:, None], -1)
        s["parent"].copy_(parent)
        s["token"].copy_(torch.where(there, at % V, -1))
        s["new_score"].copy_(best)
        s["new_done"].copy_((s["done"].bool()[parent.clamp(min=0)] | (s["token"] == end)) & there)
    return s["parent"], s["token"], s["new_score"], s["new_done"]


def _buffers(s):
    return s["k"], s["v"], s["k_scale"], s["v_scale"], s["weight"]


def _copy_pages(s, src, dst, tokens):
    """The first tokens[i] tokens of page src[i] to page dst[i], values in whole groups of 16."""
    slot = torch.arange(s["case"]["page"], device="cuda")
    keep = slot[None] < tokens[:, None]                                  # [copies, page]
    for name, mask in (("k", keep[:, None, :, None]), ("v", keep[:, None, :: 16, None, None]), ("weight", keep[:, None])):
        x = s[name].view(torch.int8) if s[name].element_size() == 1 else s[name]
        x[dst] = torch.where(mask, x[src], x[dst])
    for name in ("k_scale", "v_scale"):
        s[name][dst] = s[name][src]


def _held(pages, kv_len, P, n_pages):
    """[seqs, places]: the entries that hold cached tokens of their sequence and name a page."""
    place = torch.arange(pages.shape[1], device="cuda")
    return (place * P < kv_len[:, None]) & (pages >= 0) & (pages < n_pages)


def _run_fork(s):
    case, n_pages = s["case"], s["k"].shape[0]
    if own:
        fcp, cache = _cache(s)
        fcp.fcp_cache_fork(cache, s["pages"], s["kv_len"], s["parent"], s["news"], s["new_pages"], s["new_len"], s["counts"], s["scratch"],
                           busy=s["busy"])
    else:
        P, pages, kv_len, busy = case["page"], s["pages"].long(), s["kv_len"].long(), s["busy"].bool()
        n, width = s["new_pages"].shape
        there = (s["parent"] >= 0) & (s["parent"] < len(kv_len))
        p = s["parent"].long().clamp(0, len(kv_len) - 1)
        before = torch.where(there, kv_len[p].clamp(0, width * P), 0)
        after = (before + s["news"].clamp(min=0)).clamp(max=width * P)
        table, place = pages[p], torch.arange(width, device="cuda")
        held = _held(table, before, P, n_pages)
        # the pages that new tokens go into and earlier ones lie in
        writes = ((after > before) & (before % P > 0))[:, None] & (place == (before // P)[:, None]) & held
        reads = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
        reads[table[held & ~writes]] = True
        seq = torch.arange(n, device="cuda")[:, None].expand(n, width)
        lowest = torch.full((n_pages,), n, device="cuda").scatter_reduce_(0, table[writes], seq[writes], "amin")
        page = torch.where(held, table, 0)
        copied = writes & (reads[page] | busy[page] | (lowest[page] != seq))
        fresh = copied | ((place * P >= before[:, None]) & (place * P < after[:, None]))
        taken = busy.clone()
        taken[pages[_held(pages, kv_len, P, n_pages)]] = True
        free = torch.nonzero(~taken)[:, 0]
        rank = torch.cumsum(fresh.flatten(), 0).reshape(n, width) - 1
        got = torch.where(rank < len(free), torch.nn.functional.pad(free, (0, 1))[rank.clamp(0, len(free))], -1)
        result = torch.where(fresh, got, torch.where(held, table, -1))
        s["new_pages"].copy_(result)
        s["new_len"].copy_(after)
        moved = copied & (result >= 0)
        _copy_pages(s, table[moved], result[moved], (before % P)[:, None].expand(n, width)[moved])
        holds = busy.clone()
        holds[result[result >= 0]] = True
        need = fresh.sum()
        s["counts"].copy_(torch.stack([need.clamp(max=len(free)), (need - len(free)).clamp(min=0), n_pages - holds.sum()]))
    return (s["new_pages"], s["new_len"], s["counts"], *_buffers(s))


def _run_compact(s):
    case, n_pages = s["case"], s["k"].shape[0]
    if own:
        fcp, cache = _cache(s)
        fcp.fcp_cache_compact(cache, s["pages"], s["kv_len"], s["new_pages"], s["counts"], s["scratch"], busy=s["busy"])
    else:
        P, pages, busy = case["page"], s["pages"].long(), s["busy"].bool()
        held = _held(pages, s["kv_len"], P, n_pages)
        used = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
        used[pages[held]] = True
        stays = used & busy
        used = used & ~busy
        low = ~busy & (torch.cumsum(~busy, 0) <= used.sum())             # the lowest numbers, as many as there are pages in use
        src, dst = torch.nonzero(used & ~low)[:, 0], torch.nonzero(low & ~used)[:, 0]
        to = torch.arange(n_pages, device="cuda")
        to[src] = dst
        s["new_pages"].copy_(torch.where(held, to[torch.where(held, pages, 0)], -1))
        _copy_pages(s, src, dst, torch.full((len(src),), P, device="cuda"))
        ends = torch.nonzero(low | busy)[:, 0]
        s["counts"].copy_(torch.stack([torch.tensor(len(src), device="cuda"), used.sum() + stays.sum(), ends[-1] + 1]))
    return (s["new_pages"], s["counts"], *_buffers(s))


def _rows_of(s, name):
    """Cached rows of every sequence in 32 bits: [seqs, hkv, tokens of the longest, D] (places past a sequence's end hold anything finite)."""
    p = s["pages"].clamp(min=0).long()
    x = s[name][p]                                                       # [seqs, pages, hkv, ...]
    x = (x if name == "k" else _v_rows(x)).float() * s[name + "_scale"][p][..., None, None]
    n, m, hkv, P, D = x.shape
    return x.transpose(1, 2).reshape(n, hkv, m * P, D)


def _run_shared(s):
    case = s["case"]
    if own:
        fcp, cache = _cache(s)
        fcp.fcp_cache_attn_shared(cache, s["q"], s["cu"], s["kv_len"], s["pages"], s["groups"], s["shared"], s["scale"], s["o"], s["lse"],
                                  s["scratch"])
    else:
        n, m, hkv, D = len(s["kv_len"]), case["new"], case["hkv"], case["head_dim"]
        k = _rows_of(s, "k")
        q = s["q"].float().reshape(n, m, hkv, -1, D).permute(0, 2, 3, 1, 4)
        x = torch.matmul(q.flatten(2, 3), k.transpose(2, 3).contiguous()).reshape(n, hkv, -1, m, k.shape[2]) * s["scale"]
        last = (s["kv_len"] - m)[:, None] + torch.arange(m, device="cuda")[None]
        seen = torch.arange(k.shape[2], device="cuda") <= last[:, :, None]
        x.masked_fill_(~seen[:, None, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        p = torch.exp(x.sub_(top))
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.flatten(2, 3), _rows_of(s, "v")).reshape(n, hkv, -1, m, D) / total
        s["o"].copy_(o.permute(0, 3, 1, 2, 4).reshape(s["o"].shape))
        s["lse"].copy_((torch.log(total) + top)[..., 0].permute(1, 2, 0, 3).reshape(s["lse"].shape))
    return s["o"], s["lse"]


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------
def exact(case, seed):
    return globals()["_exact_" + case["op"]](case, prepare(case, seed))


def _exact_beam(case, s):
    """A prompt at a time on the host, the candidates of every beam put in order by (score, beam, token)."""
    B, keep, end = case["beams"], case["keep"], s["end"]
    if case["prompts"] * B * case["vocab"] > 3e7:
        return None
    score, done = s["score"].double().cpu().numpy(), s["done"].cpu().numpy()
    out = ([], [], [], [])
    for p in range(case["prompts"]):
        found = []
        for r in range(p * B, (p + 1) * B):
            if done[r]:
                found.append((-score[r], r, end, 1))
                continue
            x = s["logits"][r].double().cpu().numpy()
            lse = np.logaddexp.reduce(x[np.isfinite(x)]) if np.isfinite(x).any() else 0.0
            near = np.argsort(-x, kind="stable")[:keep]
            found += [(-(score[r] + x[t] - lse), r, int(t), int(t == end)) for t in near if np.isfinite(x[t])]
        found = sorted(found)[:keep]
        found += [(math.inf, -1, -1, 0)] * (keep - len(found))
        for o, column in zip(out, zip(*found)):
            o.append(column)
    worst, parent, token, over = (torch.tensor(o, device="cuda") for o in out)
    return parent, token, -worst.double(), over


def _doubles(s):
    """The pool's buffers in 64 bits; None for codes that are whole numbers."""
    e4m3 = s["case"]["format"] == "e4m3"
    return [s[n].double() if e4m3 or s[n].element_size() > 1 else None for n in ("k", "v", "k_scale", "v_scale", "weight")]


def _move(out, src, dst, tokens):
    for i, x in enumerate(out):
        if x is not None:
            n = (tokens, -(-tokens // 16), None, None, tokens)[i]
            if n is None:
                x[dst] = x[src]
            else:
                x[dst, :, :n] = x[src, :, :n]


def _exact_fork(case, s):
    """One sequence after the other, as a host's tables would be kept."""
    if s["new_pages"].numel() > 40000:
        return None
    P, old, lens, busy = case["page"], s["pages"].tolist(), s["kv_len"].tolist(), s["busy"].tolist()
    readers, writers = {}, {}
    tables, before, after = [], [], []
    for i, (p, new) in enumerate(zip(s["parent"].tolist(), s["news"].tolist())):
        held = old[p][: -(-lens[p] // P)]
        partly = new > 0 and lens[p] % P
        for page in held[:-1] if partly else held:
            readers[page] = True
        if partly:
            writers.setdefault(held[-1], []).append(i)
        tables.append(held)
        before.append(lens[p])
        after.append(lens[p] + new)
    in_use = {page for t, n in zip(old, lens) for page in t[: -(-n // P)]}
    free = [i for i in range(len(busy)) if not busy[i] and i not in in_use]
    out, taken = _doubles(s), 0
    for i, t in enumerate(tables):
        n = before[i]
        if after[i] > n and n % P and (t[-1] in readers or busy[t[-1]] or writers[t[-1]][0] != i):
            _move(out, t[-1], free[taken], n % P)
            t[-1] = free[taken]
            taken += 1
        while len(t) * P < after[i]:
            t.append(free[taken])
            taken += 1
    left = len(busy) - len({i for i, b in enumerate(busy) if b} | {p for t in tables for p in t})
    width = s["new_pages"].shape[1]
    return (torch.tensor([t + [-1] * (width - len(t)) for t in tables]).cuda(), torch.tensor(after).cuda(), torch.tensor([taken, 0, left]).cuda(), *out)


def _exact_compact(case, s):
    if s["k"].shape[0] > 20000:
        return None
    P, busy, width = case["page"], s["busy"].tolist(), s["pages"].shape[1]
    tables = [t[: -(-n // P)] for t, n in zip(s["pages"].tolist(), s["kv_len"].tolist())]
    used = sorted({p for t in tables for p in t if not busy[p]})
    low = [i for i, b in enumerate(busy) if not b][: len(used)]
    inside, occupied = set(low), set(used)
    holes, to, out = [i for i in low if i not in occupied], {}, _doubles(s)
    for page in used:
        if page not in inside:
            to[page] = holes[len(to)]
            _move(out, page, to[page], P)
    end = max(low + [i for i, b in enumerate(busy) if b]) + 1
    return (torch.tensor([[to.get(p, p) for p in t] + [-1] * (width - len(t)) for t in tables]).cuda(),
            torch.tensor([len(to), len({p for t in tables for p in t}), end]).cuda(), *out)


def _exact_shared(case, s):
    """A sequence at a time over its own table, with logsumexp and softmax in 64 bits."""
    group, P, cu, lens = case["hq"] // case["hkv"], case["page"], s["cu"].tolist(), s["kv_len"].tolist()
    o, lse = [], []
    for i, n in enumerate(lens):
        p = s["pages"][i, : -(-n // P)].long()
        k, v = ((s[name][p] if name == "k" else _v_rows(s[name][p])).double() * s[name + "_scale"][p].double()[..., None, None] for name in ("k", "v"))
        k, v = (x.transpose(0, 1).flatten(1, 2)[:, :n].repeat_interleave(group, 0) for x in (k, v))
        q = s["q"][cu[i]: cu[i + 1]].double()
        m = q.shape[0]
        x = torch.matmul(q.transpose(0, 1), k.transpose(1, 2).contiguous()) * s["scale"]
        x += torch.full((m, n), -math.inf, dtype=torch.float64, device="cuda").triu(n - m + 1)
        lse.append(torch.logsumexp(x, -1))
        o.append(torch.matmul(torch.softmax(x, -1), v).transpose(0, 1))
    return torch.cat(o), torch.cat(lse, 1)
