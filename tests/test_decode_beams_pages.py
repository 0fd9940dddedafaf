"""Beams whose pool has too few pages, with and without a look at the counts."""
import pytest

from paper_2602_21788_amd import binding as B


@pytest.mark.gpu
def test_tokens_that_a_step_without_a_look_lost_are_not_lost_in_silence():
    """Pages of 16 tokens, a pool of four, a prompt of 20: of four beams one goes on in the page that is begun, two get copies and one finds none.  Its new token is seen by nobody, nor are the prompt's
    last four, which lay in that page; attention is over the rest, and its next tokens would go where there is no page.  A step that looks raises for these too; one that does not goes on."""
    import torch
    from paper_2602_21788_amd.decode import BeamDecoder
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = lambda n, h: torch.randn(n, h, 64, generator=g, device="cuda").to(torch.bfloat16)
    dec = BeamDecoder(1, 4, 4, 4, 2, 2, 64, page_tokens=16, rot_dim=0)
    dec.prefill(rows(20, 2), rows(20, 2), rows(20, 2), [20])

    def step(check):
        q = rows(4, 2)
        o, lse = dec.step(q, rows(4, 2), rows(4, 2), check=check)
        ordinary = torch.empty_like(o), torch.empty_like(lse)
        work = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_ATTN, dec.cache, 4, 4, 4, 2), dtype=torch.uint8, device="cuda")
        B.fcp_cache_attn(dec.cache, q, dec._cu, dec.kv_len, dec.pages, dec.scale, *ordinary, work)
        # (two bf16 roundings of values of at most 5 or so)
        assert float((ordinary[0].float() - o.float()).abs().max()) <= 2.0 ** -6 * 5 and float((ordinary[1] - lse).abs().max()) < 1e-4

    dec.select(torch.tensor([[4.0, 3.0, 2.0, 1.0]], device="cuda"))
    with pytest.raises(MemoryError):
        step(True)
    step(False)
    pages = dec.pages.cpu().numpy()
    assert dec.counts.tolist()[:2] == [2, 1] and (pages[:3, 1] >= 0).all() and pages[3, 1] == -1 and dec.kv_len.tolist() == [21] * 4
    each = 100 * torch.eye(4, device="cuda")                 # every beam goes on
    dec.select(each)
    order = dec.chosen.tolist()
    assert sorted(order) == [0, 1, 2, 3]
    before = dec.pages.clone(), dec.kv_len.clone(), dec.steps
    with pytest.raises(MemoryError):
        step(True)
    assert torch.equal(dec.pages, before[0]) and torch.equal(dec.kv_len, before[1]) and dec.steps == before[2]
    step(False)
    assert dec.counts.tolist()[:2] == [0, 0] and dec.kv_len.tolist() == [22] * 4
    dec.select(each)
    with pytest.raises(MemoryError):
        step(True)


@pytest.mark.gpu
def test_steps_without_a_look_are_those_with_one():
    """Where there are pages enough: the same tables, codes, O and LSE."""
    import torch
    from paper_2602_21788_amd.decode import BeamDecoder
    runs = []
    for check in (True, False):
        g = torch.Generator(device="cuda").manual_seed(2)
        rows = lambda n, h: torch.randn(n, h, 64, generator=g, device="cuda").to(torch.bfloat16)
        dec = BeamDecoder(2, 3, 60, 6, 4, 2, 64, page_tokens=16)
        dec.prefill(rows(50, 4), rows(50, 2), rows(50, 2), [33, 17])
        out = []
        for t in range(20):
            dec.select(2 * torch.randn(6 if t else 2, 50, generator=g, device="cuda"))
            out += dec.step(rows(6, 4), rows(6, 2), rows(6, 2), check=check)
        runs.append(out + [dec.pages, dec.kv_len, dec.cache.k.view(torch.int8), dec.cache.v.view(torch.int8), dec.score])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
