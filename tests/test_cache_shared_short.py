"""Attention behind a common beginning where some sequences of a group have just begun: they are worked by themselves, and the others still have their beginning in common."""
import numpy as np
import pytest

from test_cache import check_attn
from test_cache_shared import Batch


def short(b, s, length, page):
    """Sequence s becomes one of `length` tokens, in a page of its own."""
    b.kv_len[s] = length
    b.pages[s] = -1
    if length:
        b.pages[s, 0] = page


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("new, hq, hkv, length", [(1, 8, 2, 1), (1, 32, 2, 1), (1, 8, 2, 32), (3, 16, 2, 3), (7, 4, 4, 0), (9, 4, 1, 40), (17, 2, 1, 48)])
@pytest.mark.parametrize("count, where", [(1, [0]), (1, [2]), (1, [4]), (1, [1, 3]), (3, [0, 4]), (5, [2])])
def test_sequences_that_have_just_begun(count, where, new, hq, hkv, length, fmt):
    """Fewer tokens than a page before the new ones, none but the new ones, fewer than there are rows.  The common pages are those of the first of the others: what the rest of them say there is
    not looked at, so that it shows whether they are worked together."""
    P, D = 32, 64 if count > 1 else 128
    b = Batch(P, D, hq, hkv, [(96 + 32 * (g % 2), [(new + i, new) for i in range(5)]) for g in range(count)], fmt)
    spare = sorted(set(range(b.ref.n_pages)) - set(b.pages[b.pages >= 0].tolist()))[0]           # (all short ones read the same page)
    for g in range(count):
        for i in where:
            short(b, 5 * g + i, length, spare)
            if length > P:
                b.pages[5 * g + i, 1] = spare
    want = b.want()
    for g in range(count):
        others = [i for i in range(5) if i not in where]
        for i in others[1:]:
            b.pages[5 * g + i, : 3 + g % 2] = -1
    check_attn(b.run(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("new, length", [(1, 1), (9, 4)])
def test_many_groups(new, length):
    """More sequences than every block looks at by itself; groups that a wave's lanes share."""
    test_sequences_that_have_just_begun(60, [0, 3], new, 4, 1, length, "int8")


@pytest.mark.gpu
def test_a_whole_page_before_the_new_rows_counts():
    """One page less a token, and one page: the first does not take part, the second bounds what is shared."""
    b = Batch(32, 64, 8, 2, [(160, [(4, 1), (5, 1), (6, 1), (7, 1)])], "int8")
    spare = [p for p in range(b.ref.n_pages) if p not in b.pages][0]
    short(b, 1, 32, spare)                                   # (31 before the new one)
    b.kv_len[2] = 33
    want = b.want()
    b.pages[2, 0] = -1                                       # the one page that is shared: read through sequence 0
    b.pages[3, 0] = -1
    check_attn(b.run(), want)


@pytest.mark.gpu
def test_rows_between_that_are_not_numbers_stay_alone():
    """The rows of a sequence that has just begun lie between the others': NaN in them reaches nobody else."""
    b = Batch(32, 64, 8, 2, [(160, [(4, 1), (5, 1), (6, 1), (7, 1)])], "int8")
    spare = [p for p in range(b.ref.n_pages) if p not in b.pages][0]
    short(b, 1, 1, spare)
    b.q[1] = np.nan
    got, want = b.run(), b.want()
    assert np.isnan(got[0][1]).all() and np.isfinite(got[0][[0, 2, 3]]).all()
    rest = lambda x: tuple(np.delete(y, 1, 0 if y.ndim == 3 else 1) if i in (0, 1, 3, 4) else y for i, y in enumerate(x))
    check_attn(rest(got), rest(want))
