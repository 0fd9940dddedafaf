"""Performance cases of the operators around a decoder's 8-bit cache, and of rotary positions:

  rotary  rotary positions of query and key rows (training: packed or sharded rows at any position; serving: new tokens),
          and the adjoint that turns fp32 gradient sums into bf16 gradients of the unrotated rows
  append  new key and value rows quantised into a paged 8-bit cache, one scale for each (page, KV head)
  attn    attention of new tokens over that cache, one token per sequence or several, optionally adding up for every
          cached token the attention weight that it got
  weigh   the same sum for the queries of a prompt whose log-sum-exp is known
  evict   the cached tokens with the least attention weight dropped, the others moved to new pages

Where `own` is false, run() computes the plain forms in elementary torch operations; where it is true, it calls the package.
Lengths follow from the case, values from the seed.  Ragged lengths: sequence i has longest / 20^frac(0.618 i) tokens.
"""
import math

import numpy as np
import torch

own = False

FARTHEST = 131072
#: (query heads, KV heads)
HEADS = [(4, 4), (8, 8), (6, 2), (10, 2), (8, 1), (32, 8), (40, 8)]


def listed():
    return [
        # the smallest calls: one new token of each of 16 sequences, rows of the fused projection's output
        {"name": "rotary_token", "op": "rotary", "rows": 16, "hq": 32, "hkv": 8, "head_dim": 128, "rot": 128, "layout": "half",
         "farthest": FARTHEST, "fused": True, "grads": False},
        # a packed training micro-batch, every query and key row
        {"name": "rotary_packed_32k", "op": "rotary", "rows": 32768, "hq": 32, "hkv": 8, "head_dim": 128, "rot": 128, "layout": "half",
         "farthest": 16384, "fused": False, "grads": False},
        # the backward of a sharded long document: a rank's fp32 sums of dQ and dK, half of the channels rotate, neighbours in pairs
        {"name": "rotary_grads_9363", "op": "rotary", "rows": 9363, "hq": 40, "hkv": 8, "head_dim": 128, "rot": 64, "layout": "pairs",
         "farthest": FARTHEST, "fused": False, "grads": True},
        # one new token of each of 64 ragged sequences
        {"name": "append_token", "op": "append", "seqs": 64, "longest": 2048, "new": 1, "hkv": 8, "head_dim": 128, "page": 64,
         "format": "e4m3"},
        # the prompts of a packed batch, straight after their forward pass
        {"name": "append_prompts", "op": "append", "seqs": 24, "longest": 4001, "new": -1, "hkv": 8, "head_dim": 128, "page": 64,
         "format": "int8"},
        # the smallest decoding step: one sequence, a small model with narrow heads
        {"name": "attn_512_d64", "op": "attn", "seqs": 1, "longest": 512, "new": 1, "hq": 4, "hkv": 4, "head_dim": 64, "page": 16,
         "format": "e4m3", "weigh": False},
        # one long document, one new token: the work has to be split over the keys
        {"name": "attn_131k", "op": "attn", "seqs": 1, "longest": 131072, "new": 1, "hq": 32, "hkv": 8, "head_dim": 128, "page": 64,
         "format": "e4m3", "weigh": False},
        # an ordinary serving batch of ragged sequences that keeps the weights for a later eviction
        {"name": "attn_64_ragged_weigh", "op": "attn", "seqs": 64, "longest": 16384, "new": 1, "hq": 32, "hkv": 8, "head_dim": 128,
         "page": 32, "format": "int8", "weigh": True},
        # the next piece of a prompt over what is cached of it
        {"name": "attn_chunk_512", "op": "attn", "seqs": 2, "longest": 16385, "new": 512, "hq": 40, "hkv": 8, "head_dim": 128, "page": 64,
         "format": "e4m3", "weigh": False},
        # the weights that a prompt's own queries give
        {"name": "weigh_4k_prompt", "op": "weigh", "seqs": 1, "longest": 4096, "hq": 8, "hkv": 8, "head_dim": 128, "page": 64,
         "format": "e4m3"},
        # a few short sequences cut to a small budget
        {"name": "evict_600_to_256", "op": "evict", "seqs": 4, "longest": 600, "budget": 256, "first": 4, "recent": 64, "hkv": 4,
         "head_dim": 64, "page": 16, "format": "int8"},
        # long documents cut to an eighth
        {"name": "evict_131k_to_16k", "op": "evict", "seqs": 4, "longest": 131072, "budget": 16384, "first": 4, "recent": 4096, "hkv": 8,
         "head_dim": 128, "page": 64, "format": "e4m3"},
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the ranges the listed ones stand for, no dearer than the dearest of them of its operator."""
    while True:
        op = rng.choice(["rotary", "rotary", "append", "append", "attn", "attn", "attn", "weigh", "evict", "evict"])
        hq, hkv = rng.choice(HEADS)
        dim = rng.choice([64, 128, 128])
        case = {"op": op, "head_dim": dim, "hkv": hkv}
        if op == "rotary":
            case.update(hq=hq, rows=_log_between(rng, 1, 40000), rot=rng.choice([dim, dim, dim // 2, dim // 4]),
                        layout=rng.choice(["half", "pairs"]), farthest=_log_between(rng, 100, 1 << 20), grads=rng.random() < 0.4)
            case["fused"] = not case["grads"] and rng.random() < 0.5
        else:
            case.update(page=rng.choice([16, 32, 64, 64, 128]), format=rng.choice(["e4m3", "int8"]))
            if op == "weigh":
                case.update(hq=hq, seqs=_log_between(rng, 1, 8), longest=_log_between(rng, 60, 4096))
            elif op == "evict":
                longest = _log_between(rng, 100, 131072)
                budget = _log_between(rng, max(24, longest // 16), longest)
                case.update(seqs=_log_between(rng, 1, 16), longest=longest, budget=budget, first=rng.randint(0, 8),
                            recent=_log_between(rng, 1, budget // 2))
            else:
                case.update(seqs=_log_between(rng, 1, 64), longest=_log_between(rng, 1, 131072),
                            new=rng.choice([1, 1, 1, _log_between(rng, 2, 512)]))
                if op == "append":
                    case["new"] = rng.choice([case["new"], -1])
                else:
                    case.update(hq=hq, weigh=rng.random() < 0.3)
        most = [work(c) for c in listed() if c["op"] == op]
        mine = work(case)
        if mine["bytes"] <= max(w["bytes"] for w in most) and mine["flops"] <= max(w["flops"] for w in most) and _padded(case) <= 1 << 31:
            return case


# ---- layouts ------------------------------------------------------------------------------------------------------------
def _lens(case):
    return [max(1, int(case["longest"] / 20 ** ((0.618 * i) % 1))) for i in range(case["seqs"])]


def _news(case):
    """New tokens of every sequence (they are the last ones of its length)."""
    new = case.get("new", -1)
    return [n if new < 0 else min(n, new) for n in _lens(case)]


def _padded(case):
    """Elements of a rectangle that holds all keys, or all scores: what the plain form needs at once."""
    if case["op"] == "rotary":
        return 0
    L, n = case["longest"], max(_news(case))
    return case["seqs"] * max(L * case["hkv"] * case["head_dim"], case.get("hq", 0) * n * L)


def _pairs(case):
    return sum(n * (2 * L - n + 1) // 2 for L, n in zip(_lens(case), _news(case)))


def work(case):
    """What the operator cannot do without: inputs read once, outputs written once, and the products."""
    D, hkv = case["head_dim"], case["hkv"]
    if case["op"] == "rotary":
        elements = case["rows"] * (case["hq"] + hkv) * D
        return {"bytes": elements * ((4 if case["grads"] else 2) + 2) + 4 * case["rows"],
                "flops": 3 * case["rows"] * (case["hq"] + hkv) * case["rot"]}
    keys, new = sum(_lens(case)), sum(_news(case))
    scales = 8 * hkv * sum(-(-n // case["page"]) for n in _lens(case))
    if case["op"] == "append":
        return {"bytes": 2 * new * hkv * D * 3, "flops": 2 * new * hkv * D * 2}
    if case["op"] == "evict":
        kept = sum(min(n, case["budget"]) for n in _lens(case))
        return {"bytes": 4 * hkv * (keys + 2 * kept) + 2 * 2 * kept * hkv * D, "flops": 2 * kept * hkv * D * 2}
    rows = new * case["hq"]
    if case["op"] == "weigh":
        return {"bytes": keys * hkv * (D + 8) + rows * (2 * D + 4) + scales // 2, "flops": 2 * _pairs(case) * D * case["hq"]}
    return {"bytes": keys * hkv * (2 * D + (8 if case["weigh"] else 0)) + rows * (4 * D + 4) + scales,
            "flops": 4 * _pairs(case) * D * case["hq"]}


# ---- inputs -------------------------------------------------------------------------------------------------------------
LEAST = -110                                  # least exponent of a scale


def _exponent(amax, fmt):
    """Least e with amax <= most * 2^e, for the format's largest value: 448 = 0.875 * 2^9, 127 = (127 / 128) * 2^7."""
    m, x = torch.frexp(amax)
    part, bits = (0.875, 9) if fmt == "e4m3" else (127 / 128, 7)
    return torch.where(amax > 0, x - bits + (m > part).int(), LEAST).clamp(min=LEAST)


def _encode(x, e, fmt):
    """x in units of 2^e, rounded to the nearest value of the format."""
    x = torch.ldexp(x, -e)
    return x.to(torch.float8_e4m3fn) if fmt == "e4m3" else x.round().clamp(-127, 127).to(torch.int8)


def _v_pages(v):
    """Value rows [..., page, D] in the cache's order [..., page / 16, D, 16]."""
    *lead, P, D = v.shape
    return v.reshape(*lead, P // 16, 16, D).transpose(-1, -2)


def _v_rows(v):
    """The reverse of _v_pages."""
    *lead, n, D, _ = v.shape
    return v.transpose(-1, -2).reshape(*lead, n * 16, D)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _rows(gen, n, heads, dim):
    """bf16 rows as projections give them: normal, a few channels and a few tokens larger."""
    x = _normal(gen, n, heads, dim)
    x[:, :, :: 32] *= 3
    return (x * torch.exp(0.3 * _normal(gen, n, 1, 1))).to(torch.bfloat16)


def _pool(gen, case, n_pages):
    """A cache of n_pages pages whose every slot holds a token."""
    shape = (n_pages, case["hkv"], case["page"], case["head_dim"])
    pool = {}
    for name in ("k", "v"):
        x = _normal(gen, *shape)
        x[..., :: 32] *= 3
        e = _exponent(x.abs().amax((2, 3)), case["format"])
        codes = _encode(x, e[:, :, None, None], case["format"])
        pool[name] = (codes if name == "k" else _v_pages(codes)).contiguous()
        pool[name + "_scale"] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
        del x, codes
    # what many steps of decoding leave: heavy-tailed, the newest tokens with little or nothing, many equal
    pool["weight"] = (torch.exp(2 * _normal(gen, *shape[:3])) * 64).floor() / 64
    return pool


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    D, hkv = case["head_dim"], case["hkv"]
    if case["op"] == "rotary":
        n, hq = case["rows"], case["hq"]
        s = {"case": case, "pos": torch.randint(0, case["farthest"], (n,), generator=gen, device="cuda", dtype=torch.int32)}
        half = case["rot"] // 2
        s["turns"] = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half) / (2 * math.pi)
        if case["grads"]:
            s["q"], s["k"] = _normal(gen, n, hq, D), _normal(gen, n, hkv, D)
        elif case["fused"]:
            qkv = _rows(gen, n, hq + 2 * hkv, D)
            s["q"], s["k"] = qkv[:, :hq], qkv[:, hq: hq + hkv]
        else:
            s["q"], s["k"] = _rows(gen, n, hq, D), _rows(gen, n, hkv, D)
        s["q_out"] = torch.empty(n, hq, D, dtype=torch.bfloat16, device="cuda")
        s["k_out"] = torch.empty(n, hkv, D, dtype=torch.bfloat16, device="cuda")
        return s
    P, lens, news = case["page"], _lens(case), _news(case)
    counts = [-(-n // P) for n in lens]
    order = np.random.RandomState(seed % (1 << 32)).permutation(sum(counts))          # pages of a cache in use lie anywhere
    table = np.full((len(lens), max(counts)), -1, np.int32)
    at = np.concatenate([[0], np.cumsum(counts)])
    for i, c in enumerate(counts):
        table[i, :c] = order[at[i]: at[i + 1]]
    kept = [min(n, case["budget"]) for n in lens] if case["op"] == "evict" else []
    new_counts = [-(-n // P) for n in kept]
    s = {"case": case, "kv_len": _int(lens), "pages": torch.from_numpy(table).cuda(),
         "cu": _int(np.concatenate([[0], np.cumsum(news)]).tolist())}
    s.update(_pool(gen, case, sum(counts) + sum(new_counts)))
    scale = s["scale"] = 1 / math.sqrt(D)
    if case["op"] == "append":
        s["k_new"], s["v_new"] = _rows(gen, sum(news), hkv, D), _rows(gen, sum(news), hkv, D)
        # which pages are written, from which slot on, and the page and slot of every new row
        touched, first, row_page, row_slot = [], [], [], []
        for i, (n, m) in enumerate(zip(lens, news)):
            for p in range((n - m) // P, (n - 1) // P + 1):
                lo = max(n - m, p * P)
                row_page += [len(touched)] * (min(n, (p + 1) * P) - lo)
                row_slot += range(lo - p * P, min(n, (p + 1) * P) - p * P)
                touched.append(int(table[i, p]))
                first.append(lo - p * P)
        s["plan"] = [torch.tensor(x, dtype=torch.int64, device="cuda") for x in (touched, first, row_page, row_slot)]
    elif case["op"] == "evict":
        # the new pages are the pool's last ones, empty so far
        s["n_old"] = sum(counts)
        for name in ("k", "v", "k_scale", "v_scale", "weight"):
            x = s[name][s["n_old"]:]
            (x.view(torch.int8) if x.element_size() == 1 else x).zero_()
        order = np.random.RandomState(seed % (1 << 32) + 1).permutation(sum(new_counts)) + s["n_old"]
        table = np.full((len(lens), max(new_counts)), -1, np.int32)
        at = np.concatenate([[0], np.cumsum(new_counts)])
        for i, c in enumerate(new_counts):
            table[i, :c] = order[at[i]: at[i + 1]]
        s["new_pages"] = torch.from_numpy(table).cuda()
        s["new_of"] = torch.tensor([[i, j] for i, c in enumerate(new_counts) for j in range(c)], device="cuda")   # [new pages in use, 2]
        s["kept"] = torch.empty(len(lens), hkv, case["budget"], dtype=torch.int32, device="cuda")
        s["new_len"] = torch.empty(len(lens), dtype=torch.int32, device="cuda")
    else:
        hq = case["hq"]
        s["q"] = _rows(gen, sum(news), hq, D)
        s["o"] = torch.empty(sum(news), hq, D, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(hq, sum(news), dtype=torch.float32, device="cuda")
        # the row of the packed queries that is token j of sequence i, and which of these there are
        j = torch.arange(max(news), device="cuda")
        s["there"] = j[None] < torch.diff(s["cu"])[:, None]
        s["row"] = torch.where(s["there"], s["cu"][:-1, None] + j[None], 0)
        if case["op"] == "weigh":
            s["lse"].copy_(_lse(s, _scores(s)))
    return s


# ---- the operators ------------------------------------------------------------------------------------------------------
def _cache(s):
    """The package's view of the cache in `s`, and work space of the size it asks for: made once."""
    import paper_2602_21788_amd as fcp
    if "cache" not in s:
        c = s["case"]
        s["cache"] = fcp.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["weight"])
        which = {"attn": fcp.FCP_SCRATCH_CACHE_WEIGH if c.get("weigh") else fcp.FCP_SCRATCH_CACHE_ATTN, "evict": fcp.FCP_SCRATCH_CACHE_EVICT}.get(c["op"])
        if which is not None:
            n = fcp.fcp_cache_scratch_bytes(which, s["cache"], c["seqs"], s["pages"].shape[1], s["q"].shape[0] if "q" in s else 0, c.get("hq", c["hkv"]))
            s["scratch"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return fcp, s["cache"]


def _rotary(x, c, sn, case):
    """Pairs of the first `rot` channels turned by the angles, the others as they are."""
    rot, x = case["rot"], x.float()
    a, b = (x[..., : rot // 2], x[..., rot // 2: rot]) if case["layout"] == "half" else (x[..., 0: rot: 2], x[..., 1: rot: 2])
    ya, yb = a * c - b * sn, a * sn + b * c
    y = torch.cat((ya, yb), -1) if case["layout"] == "half" else torch.stack((ya, yb), -1).flatten(-2)
    return torch.cat((y, x[..., rot:]), -1).to(torch.bfloat16)


def _rows_of(s, name):
    """Cached rows of every sequence in 32 bits: [seqs, hkv, tokens of the longest, D] (places past a sequence's end hold anything finite)."""
    p = s["pages"].clamp(min=0).long()
    x = s[name][p]                                                       # [seqs, pages, hkv, ...]
    x = (x if name == "k" else _v_rows(x)).float() * s[name + "_scale"][p][..., None, None]
    n, m, hkv, P, D = x.shape
    return x.transpose(1, 2).reshape(n, hkv, m * P, D)


def _scores(s):
    """Scaled scores [seqs, hkv, query heads of a KV head, new tokens, tokens], -inf where a token is not seen."""
    case, k = s["case"], _rows_of(s, "k")
    n, m = s["row"].shape
    q = s["q"][s["row"].long()].float().reshape(n, m, case["hkv"], -1, case["head_dim"]).permute(0, 2, 3, 1, 4)
    x = torch.matmul(q.flatten(2, 3), k.transpose(2, 3)).reshape(n, case["hkv"], -1, m, k.shape[2]) * s["scale"]
    last = (s["kv_len"] - torch.diff(s["cu"]))[:, None] + torch.arange(m, device="cuda")[None]
    seen = (torch.arange(k.shape[2], device="cuda") <= last[:, :, None]) & s["there"][:, :, None]
    return x.masked_fill_(~seen[:, None, None], -math.inf)


def _packed(s, x):
    """[seqs, hkv, group, new tokens, ...] of the tokens that there are: [rows, heads, ...]."""
    return x.movedim(3, 1)[s["there"]].flatten(1, 2)


def _lse(s, x):
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    return _packed(s, (torch.log((x - top).exp_().sum(-1)) + top[..., 0])).T.contiguous()


def _add_weight(s, p):
    """p: probabilities [seqs, hkv, group, new tokens, tokens], added up over the rows into the pages."""
    P, n = s["case"]["page"], s["case"]["seqs"]
    got = p.sum((2, 3))                                                  # [seqs, hkv, tokens]
    got = got.reshape(n, got.shape[1], -1, P).transpose(1, 2)            # [seqs, pages, hkv, P]
    there = s["pages"] >= 0
    s["weight"][s["pages"][there].long()] += got[there]


def run(s):
    return globals()["_run_" + s["case"]["op"]](s)


def _run_rotary(s):
    case = s["case"]
    if own:
        import paper_2602_21788_amd as fcp
        fcp.fcp_rotary([(s["q"], s["q_out"], s["pos"]), (s["k"], s["k_out"], s["pos"])], s["turns"], case["rot"],
                       fcp.FCP_ROTARY_HALF if case["layout"] == "half" else fcp.FCP_ROTARY_PAIRS, backward=case["grads"])
        return s["q_out"], s["k_out"]
    t = s["pos"].double()[:, None] * s["turns"]
    angle = (t - t.round()) * (2 * math.pi) * (-1 if case["grads"] else 1)
    c, sn = angle.cos().float()[:, None], angle.sin().float()[:, None]
    return _rotary(s["q"], c, sn, case), _rotary(s["k"], c, sn, case)


def _append(s, name):
    case, (touched, first, row_page, row_slot) = s["case"], s["plan"]
    fmt, x = case["format"], s[name + "_new"].float()                    # [rows, hkv, D]
    n, hkv = len(touched), case["hkv"]
    amax = torch.zeros(n, hkv, device="cuda").scatter_reduce_(0, row_page[:, None].expand(-1, hkv), x.abs().amax(-1), "amax")
    e, before = _exponent(amax, fmt), torch.frexp(s[name + "_scale"][touched])[1] - 1
    e = torch.where(first[:, None] > 0, torch.maximum(e, before), e)
    old = s[name][touched]
    codes = old if name == "k" else _v_rows(old)
    lives = (torch.arange(case["page"], device="cuda") < first[:, None])[:, None, :, None]
    back = torch.where(lives, codes.float(), 0.0)
    kept = _encode(torch.ldexp(back, before[:, :, None, None]), e[:, :, None, None], fmt)
    bits = torch.where(lives, kept.view(torch.int8), codes.view(torch.int8))
    bits[row_page, :, row_slot] = _encode(x, e[row_page][:, :, None], fmt).view(torch.int8)
    s[name].view(torch.int8)[touched] = bits if name == "k" else _v_pages(bits)
    s[name + "_scale"][touched] = torch.ldexp(torch.ones_like(amax), e)
    if name == "k":
        s["weight"].transpose(1, 2)[touched[row_page], row_slot] = 0


def _run_append(s):
    if own:
        fcp, cache = _cache(s)
        fcp.fcp_cache_append(cache, s["k_new"], s["v_new"], s["cu"], s["kv_len"], s["pages"])
    else:
        _append(s, "k")
        _append(s, "v")
    return s["k"], s["v"], s["k_scale"], s["v_scale"], s["weight"]


def _run_attn(s):
    weigh = s["case"]["weigh"]
    if own:
        fcp, cache = _cache(s)
        fcp.fcp_cache_attn(cache, s["q"], s["cu"], s["kv_len"], s["pages"], s["scale"], s["o"], s["lse"], s["scratch"], weigh=weigh)
    else:
        x = _scores(s)
        top = x.amax(-1, keepdim=True).clamp(min=-1e30)
        p = torch.exp(x.sub_(top))
        total = p.sum(-1, keepdim=True)
        p = p.div_(total.clamp(min=1e-30))
        o = torch.matmul(p.flatten(2, 3), _rows_of(s, "v")).reshape(*p.shape[:4], -1)
        s["o"].copy_(_packed(s, o))
        s["lse"].copy_(_packed(s, torch.log(total[..., 0]) + top[..., 0]).T)
        if weigh:
            _add_weight(s, p)
    return (s["o"], s["lse"], s["weight"]) if weigh else (s["o"], s["lse"])


def _run_weigh(s):
    if own:
        fcp, cache = _cache(s)
        fcp.fcp_cache_weigh(cache, s["q"], s["lse"], s["cu"], s["kv_len"], s["pages"], s["scale"])
    else:
        case, (n, m) = s["case"], s["row"].shape
        lse = s["lse"].T[s["row"].long()].reshape(n, m, case["hkv"], -1).permute(0, 2, 3, 1)
        _add_weight(s, torch.exp(_scores(s).sub_(lse[..., None])))
    return s["weight"]


def _run_evict(s):
    case = s["case"]
    if own:
        fcp, cache = _cache(s)
        fcp.fcp_cache_evict(cache, s["pages"], s["kv_len"], s["new_pages"], case["budget"], case["first"], case["recent"], s["kept"],
                            s["new_len"], s["scratch"])
    else:
        P, B, hkv, budget, fmt = case["page"], case["seqs"], case["hkv"], case["budget"], case["format"]
        p = s["pages"].clamp(min=0).long()
        w = s["weight"][p].transpose(1, 2).reshape(B, hkv, -1)           # [seqs, hkv, tokens]
        t, n = torch.arange(w.shape[2], device="cuda"), s["kv_len"][:, None]
        w = w.masked_fill(((t < case["first"]) | (t >= n - case["recent"]))[:, None], math.inf).masked_fill((t >= n)[:, None], -math.inf)
        at = w.sort(dim=-1, descending=True, stable=True)[1][..., :budget]
        n_new = s["kv_len"].clamp(max=budget)
        there = (torch.arange(at.shape[2], device="cuda") < n_new[:, None])[:, None]
        at = torch.where(there, at, w.shape[2]).sort(dim=-1)[0]
        s["kept"].fill_(-1)[..., : at.shape[2]] = torch.where(there, at, -1).int()
        s["new_len"].copy_(n_new)
        # the kept slots of every new page: [pages in use, hkv, P]
        row, j = s["new_of"].unbind(1)
        slot = j[:, None] * P + torch.arange(P, device="cuda")
        lives = (slot < n_new.long()[row][:, None])[:, None]
        src = torch.where(lives, at[row[:, None], :, slot.clamp(max=at.shape[2] - 1)].transpose(1, 2), 0)
        page, head, slot = p[row[:, None, None], src // P], torch.arange(hkv, device="cuda")[:, None], src % P
        new = s["new_pages"][row, j].long()
        for name in ("k", "v"):
            x = s["k"][page, head, slot] if name == "k" else s["v"].transpose(3, 4)[page, head, slot // 16, slot % 16]
            x = x.float() * s[name + "_scale"][page, head][..., None] * lives[..., None]
            e = _exponent(x.abs().amax((2, 3)), fmt)
            x = _encode(x, e[..., None, None], fmt)
            s[name].view(torch.int8)[new] = (x if name == "k" else _v_pages(x)).view(torch.int8)
            s[name + "_scale"][new] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
        s["weight"][new] = s["weight"][page, head, slot] * lives
    a = s["n_old"]
    return s["k"][a:], s["v"][a:], s["k_scale"][a:], s["v_scale"][a:], s["weight"][a:], s["kept"], s["new_len"]


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------
def exact(case, seed):
    return globals()["_exact_" + case["op"]](case, prepare(case, seed))


def _exact_rotary(case, s):
    """y = x e^(i angle) on the pairs taken as complex numbers; the adjoint turns back."""
    rot = case["rot"]
    angle = s["pos"].double()[:, None] * s["turns"] * (2 * math.pi)
    turn = torch.polar(torch.ones_like(angle), -angle if case["grads"] else angle)[:, None]
    out = []
    for x in (s["q"].double(), s["k"].double()):
        y = x.clone()
        if case["layout"] == "half":
            z = torch.complex(x[..., : rot // 2], x[..., rot // 2: rot]) * turn
            y[..., : rot // 2], y[..., rot // 2: rot] = z.real, z.imag
        else:
            z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], -1, 2)) * turn
            y[..., :rot] = torch.view_as_real(z).flatten(-2)
        out.append(y)
    return tuple(out)


def _most(case):
    return 448.0 if case["format"] == "e4m3" else 127.0


def _nearest(x, fmt):
    """The format's value nearest to x (64 bits, at most the largest one): the spacing of e4m3 is 2^(exponent - 3), 2^-9 at least."""
    if fmt == "int8":
        return x.round()
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return (x / step).round() * step


def _least_scale(amax, case):
    """The least power of two, 2^LEAST or more, in whose units amax is within the format."""
    e = math.ceil(math.log2(amax / _most(case))) if amax > 0 else LEAST
    e += 1 if amax > _most(case) * 2.0 ** e else 0
    e -= 1 if amax > 0 and amax <= _most(case) * 2.0 ** (e - 1) else 0
    return 2.0 ** max(e, LEAST)


def _exact_append(case, s):
    if sum(_news(case)) * case["hkv"] > 4096:            # one (page, head) at a time: quick for the small cases only
        return None
    touched, first, row_page, row_slot = (t.tolist() for t in s["plan"])
    out = []
    for name in ("k", "v"):
        codes = s[name].double()
        codes = codes if name == "k" else _v_rows(codes)
        scales = s[name + "_scale"].double()
        for t, (page, lo) in enumerate(zip(touched, first)):
            rows = [r for r, p in enumerate(row_page) if p == t]
            slots = [row_slot[r] for r in rows]
            x = s[name + "_new"][rows].double()                          # [rows, hkv, D]
            for h in range(case["hkv"]):
                scale = _least_scale(float(x[:, h].abs().max()), case)
                if lo:
                    scale = max(scale, float(scales[page, h]))
                    codes[page, h, :lo] = _nearest(codes[page, h, :lo] * scales[page, h] / scale, case["format"])
                codes[page, h, slots] = _nearest(x[:, h] / scale, case["format"])
                scales[page, h] = scale
        out.append((codes if name == "k" else _v_pages(codes).contiguous(), scales))
    weight = s["weight"].double()
    for r, t in enumerate(row_page):
        weight[touched[t], :, row_slot[r]] = 0
    codes = [c if case["format"] == "e4m3" else None for c, _ in out]
    return (*codes, out[0][1], out[1][1], weight)


def _of_sequence(s, name, i):
    """[hkv, tokens, D] of sequence i in 64 bits."""
    n, P = int(s["kv_len"][i]), s["case"]["page"]
    p = s["pages"][i, : -(-n // P)].long()
    x = s[name][p].double()
    x = (x if name == "k" else _v_rows(x)) * s[name + "_scale"][p].double()[..., None, None]
    return x.transpose(0, 1).flatten(1, 2)[:, :n]


def _exact_attention(case, s, with_o):
    group, cu = case["hq"] // case["hkv"], s["cu"].tolist()
    o, lse, weight = [], [], s["weight"].double()
    for i, n in enumerate(_lens(case)):
        q, k = s["q"][cu[i]: cu[i + 1]].double(), _of_sequence(s, "k", i)
        m = q.shape[0]
        x = torch.matmul(q.transpose(0, 1), k.repeat_interleave(group, 0).transpose(1, 2)) * s["scale"]      # [hq, m, n]
        x += torch.full((m, n), -math.inf, dtype=torch.float64, device="cuda").triu(n - m + 1)
        lse.append(torch.logsumexp(x, -1))
        p = torch.softmax(x, -1) if with_o else torch.exp(x - s["lse"][:, cu[i]: cu[i + 1], None].double())
        if with_o:
            o.append(torch.matmul(p, _of_sequence(s, "v", i).repeat_interleave(group, 0)).transpose(0, 1))
        got = p.sum(1).reshape(case["hkv"], group, n).sum(1)
        for j in range(-(-n // case["page"])):
            part = got[:, j * case["page"]: (j + 1) * case["page"]]
            weight[int(s["pages"][i, j]), :, : part.shape[1]] += part
    return (torch.cat(o) if with_o else None), torch.cat(lse, 1), weight


def _exact_attn(case, s):
    o, lse, weight = _exact_attention(case, s, True)
    return (o, lse, weight) if case["weigh"] else (o, lse)


def _exact_weigh(case, s):
    return _exact_attention(case, s, False)[2]


def _exact_evict(case, s):
    if case["seqs"] * case["hkv"] * case["budget"] > 65536:             # one (page, head) at a time
        return None
    P, kept_to, weight = case["page"], s["new_pages"].tolist(), s["weight"].double()
    codes, scales = {"k": s["k"].double(), "v": _v_rows(s["v"].double())}, {n: s[n + "_scale"].double() for n in ("k", "v")}
    for i, n in enumerate(_lens(case)):
        old = s["pages"][i, : -(-n // P)].long()
        w = s["weight"][old].transpose(0, 1).flatten(1, 2)[:, :n].double().cpu().numpy()
        rows = {name: _of_sequence(s, name, i) for name in ("k", "v")}
        for h in range(case["hkv"]):
            order = sorted(range(n), key=lambda t: (not (t < case["first"] or t >= n - case["recent"]), -w[h, t], t))
            keep = sorted(order[: case["budget"]])
            for j in range(-(-len(keep) // P)):
                at, page = keep[j * P: (j + 1) * P], kept_to[i][j]
                for name in ("k", "v"):
                    x = rows[name][h, at]
                    scale = scales[name][page, h] = _least_scale(float(x.abs().max()), case)
                    codes[name][page, h].zero_()[: len(at)] = _nearest(x / scale, case["format"])
                weight[page, h].zero_()[: len(at)] = torch.from_numpy(w[h, at])
    a, e4m3 = s["n_old"], case["format"] == "e4m3"
    return (codes["k"][a:] if e4m3 else None, _v_pages(codes["v"][a:]).contiguous() if e4m3 else None, scales["k"][a:], scales["v"][a:],
            weight[a:], None, None)
