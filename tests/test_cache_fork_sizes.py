"""fcp_cache_fork: sizes whose counts would not fit 32 bits, and what is accepted just below (on the CPU)."""
import pytest

from paper_2602_21788_amd import binding as B
from test_cache_fork import Call


@pytest.mark.parametrize("n_new, max_pages", [(300, 1 << 23), (257, 1 << 23), (256, 1 << 23), (1 << 20, 1 << 11), ((1 << 11) + 1, 1 << 20)])
def test_new_tables_of_2_to_the_31_entries_are_refused(n_new, max_pages):
    """Sequences may all need as many pages as their tables have entries; pages are counted in 32 bits."""
    c = Call(hkv=1, page_tokens=16).c
    assert n_new * max_pages >= 1 << 31
    with pytest.raises(B.FcpError, match="2\\^31"):
        B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_FORK, c, n_new, max_pages)
    for n_seqs in (0, 2):                                    # (one block marks and plans where there are few old entries, several launches else)
        assert Call(hkv=1, page_tokens=16, n_seqs=n_seqs, n_new=n_new, max_pages=max_pages).fork() == B.FCP_ERR_UNSUPPORTED
        assert b"2^31" in B.lib().fcp_last_error()


def test_sizes_below_are_accepted():
    c = Call(hkv=1, page_tokens=16).c
    assert B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_FORK, c, 255, 1 << 23) > 0
    # a table of this step may be larger: its entries are not added up
    assert Call(hkv=1, page_tokens=16, n_seqs=300, n_new=3, max_pages=1 << 23, bytes=0).fork() == B.FCP_ERR_CAPACITY
