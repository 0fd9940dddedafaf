"""Selection, fork, compaction, attention behind a common beginning: outputs that lie on inputs or on each other, and addresses that are no integer's, are refused (on the CPU)."""
import pytest

from paper_2602_21788_amd import binding as B
from test_cache_fork import Call

AT = 1 << 20                                                 # far from the other addresses, which nobody looks at


def refused(rc, *words):
    assert rc == B.FCP_ERR_INVALID_ARG, (rc, B.lib().fcp_last_error())
    assert all(w.encode() in B.lib().fcp_last_error() for w in words), B.lib().fcp_last_error()


# sequences 2 -> 4, tables of 3 pages, 9 pages: pages 24 bytes, kv_len 8, parent and news 16, busy 9, new_pages 48, new_len 16, counts 12
FORK = dict(pages=AT, kv_len=AT + 0x100, parent=AT + 0x200, news=AT + 0x300, busy=AT + 0x400, new_pages=AT + 0x500, new_len=AT + 0x600, counts=AT + 0x700, scratch=AT + 0x100000)
FORK_BYTES = dict(pages=24, kv_len=8, parent=16, news=16, busy=9, new_pages=48, new_len=16, counts=12)


@pytest.mark.parametrize("out", ["new_pages", "new_len", "counts"])
@pytest.mark.parametrize("other", list(FORK_BYTES))
def test_fork(out, other):
    if out == other:
        return
    for at in (0, -FORK_BYTES[out] + 4, (FORK_BYTES[other] - 1) // 4 * 4):             # the same beginning; the last of one on the first of the other, both ways round
        refused(Call(**{**FORK, out: FORK[other] + at}).fork(), "fcp_cache_fork", "apart")
    # next to each other is apart: the scratch is what is refused then
    for at in (-FORK_BYTES[out], (FORK_BYTES[other] + 3) // 4 * 4):
        assert Call(**{**FORK, out: FORK[other] + at, "bytes": 0}).fork() == B.FCP_ERR_CAPACITY


def test_fork_scratch():
    need = B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_FORK, Call().c, 4, 3)
    for name in FORK_BYTES:
        refused(Call(**{**FORK, "scratch": FORK[name] // 256 * 256, "bytes": need}).fork(), "scratch")
    for name in ("pages", "kv_len", "parent", "news", "new_pages", "new_len", "counts"):
        refused(Call(**{**FORK, name: FORK[name] + 2}).fork(), "aligned")


# tables of 2 x 3
COMPACT = dict(pages=AT, kv_len=AT + 0x100, busy=AT + 0x200, new_pages=AT + 0x300, counts=AT + 0x400, scratch=AT + 0x100000)
COMPACT_BYTES = dict(pages=24, kv_len=8, busy=9, new_pages=24, counts=12)


@pytest.mark.parametrize("out", ["new_pages", "counts"])
@pytest.mark.parametrize("other", list(COMPACT_BYTES))
def test_compact(out, other):
    if out == other:
        return
    for at in (0, -COMPACT_BYTES[out] + 4, (COMPACT_BYTES[other] - 1) // 4 * 4):
        if (out, other, at) != ("new_pages", "pages", 0):    # (the table itself)
            refused(Call(**{**COMPACT, out: COMPACT[other] + at}).compact(), "fcp_cache_compact", "apart")
    for name in ("pages", "kv_len", "new_pages", "counts"):
        refused(Call(**{**COMPACT, name: COMPACT[name] + 1}).compact(), "aligned")


# 2 prompts of 3 beams, 6 kept, 100 logits a row, rows 128 apart
BEAM = dict(logits=AT, score=AT + 0x10000, done=AT + 0x10100, parent=AT + 0x10200, token=AT + 0x10300, new_score=AT + 0x10400, new_done=AT + 0x10500, scratch=AT + 0x20000)
BEAM_BYTES = dict(score=24, done=6, parent=48, token=48, new_score=48, new_done=12)


def beam(**kw):
    a = {**BEAM, "type": B.FCP_F32, "bytes": 1 << 30, **kw}
    return B.lib().fcp_beam_select(a["logits"], a["type"], 128, 2, 3, 100, a["score"], a["done"], 5, 6, a["parent"], a["token"], a["new_score"], a["new_done"], a["scratch"], a["bytes"], None)


@pytest.mark.parametrize("out", ["parent", "token", "new_score", "new_done"])
@pytest.mark.parametrize("other", list(BEAM_BYTES))
def test_select(out, other):
    if out == other:
        return
    for at in (0, (-BEAM_BYTES[out] + 4) // 4 * 4, (BEAM_BYTES[other] - 1) // 4 * 4):
        refused(beam(**{out: BEAM[other] + at}), "fcp_beam_select", "apart")


def test_select_on_logits_and_scratch():
    row, used = 512, 400
    for at in (0, used - 4, row, 5 * row + used - 4, -44, 3 * row - 4, 2 * row + used - 4):
        refused(beam(parent=AT + at), "apart")
    need = B.fcp_beam_scratch_bytes(2, 3, 100, 6)
    refused(beam(scratch=BEAM["score"] - need // 256 * 256 + 256, bytes=need), "apart")
    # between two rows is apart, behind the last row too: the scratch is what is refused then
    for at in (used, row - 48, 4 * row + used, 5 * row + used):
        assert beam(parent=AT + at, bytes=0) == B.FCP_ERR_CAPACITY


def test_attention_behind_a_common_beginning():
    from test_cache_shared import _call
    for kw in (dict(groups=0x10002), dict(shared=0x10001)):
        refused(_call(**kw), "fcp_cache_attn_shared", "aligned")
