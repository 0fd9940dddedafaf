"""The training path of a rank with rotary positions: forward and gradients against the 64-bit oracle on the rotated rows, gradients of the rows before by the adjoint
in 64 bits, both ways of finishing the backward, and a graph."""
import numpy as np
import pytest

import fcp_synth as synth
from oracle import attn as oattn
from oracle import plan as oplan
from paper_2602_21788_amd import binding as B

rel = lambda a, b: float(np.abs(a - b).max() / np.abs(b).max())


def turn(x, pos, turns, rot, sign):
    """Half layout in 64 bits."""
    a = 2 * np.pi * sign * (pos.astype(np.float64)[:, None] * turns)
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    y = x.copy()
    u, v = x[..., : rot // 2], x[..., rot // 2: rot]
    y[..., : rot // 2], y[..., rot // 2: rot] = u * c - v * s, u * s + v * c
    return y


@pytest.mark.gpu
@pytest.mark.parametrize("D,rot,spans", [(128, 128, None), (64, 32, None), (128, 64, [(0, 100, 200)])])
def test_rotated_training_pass(D, rot, spans):
    import torch
    from paper_2602_21788_amd.rank import RankAttention, dev_to_bits
    wl = synth.custom_workload([700, 150, 33], [3, 1, 1], hq=8, hkv=2, head_dim=D, rank=1, seed=5)
    q, k, v, do = synth.draw_qkvdo(wl)
    ra = RankAttention(wl.seq_lens, wl.cp_degree, 1, 8, 2, D, wl.softmax_scale, spans=spans)
    turns, _ = B.fcp_rotary_frequencies(rot, 10000.0, B.FCP_ROTARY_LINEAR, 2.0)
    ra.set_rotary(turns, rot)
    ra.set_inputs(q, k, v, do)
    # positions: the rank's chunks' own numbers
    want = np.concatenate([np.arange(c["seq_start"], c["seq_start"] + c["len"]) for c in ra.my_chunks])
    assert np.array_equal(ra.q_pos.cpu().numpy(), want)
    ra.rotate_inputs()
    pos_k = ra.k_pos.cpu().numpy()
    f64 = synth.bf16_bits_to_f64
    # one rounding to bf16 (half a step: 2^-8 of the value, by the rule for tolerances) and the kernel's products, 6e-7 of two channels' magnitudes
    for got, x, pos in ((ra.q, q[ra.rows], want), (ra.k, k, pos_k)):
        y = turn(f64(x), pos, turns, rot, 1)
        assert (np.abs(f64(dev_to_bits(got)) - y) <= 2.0 ** -8 * np.abs(y) + 6e-7 * 2 * np.abs(f64(x)).max()).all()
    # the rotated rows as the oracle's inputs
    kr = dev_to_bits(ra.k)
    qr = q.copy()
    qr[ra.rows] = dev_to_bits(ra.q)
    ra.forward()
    ra.zero_grads()
    ra.backward_delta()
    ra.backward_steps()
    ra.finalize()
    dq_turned, dk_turned = f64(dev_to_bits(ra.dq)), f64(dev_to_bits(ra.dk))
    ra.finalize_rotary()
    dq, dk = f64(dev_to_bits(ra.dq)), f64(dev_to_bits(ra.dk))
    # the gradients of the rows before are the adjoint of the others', which come rounded here: half a step of both roundings, 2^-8 each, on two channels
    for a, b, pos in ((dq, dq_turned, want), (dk, dk_turned, pos_k)):
        y = turn(b, pos, turns, rot, -1)
        assert np.abs(a - y).max() <= 3 * 2.0 ** -8 * np.abs(b).max()
    if spans is None:
        rows = oplan.rank_rows(oplan.shard_plan(wl.seq_lens, wl.cp_degree)[0], wl.cu_seqlens, 1)
        O, LSE = oattn.attn_fwd(qr, kr, v, wl.cu_seqlens, wl.softmax_scale, rows)
        dQ = oattn.attn_dq(qr, kr, v, do, wl.cu_seqlens, wl.softmax_scale, rows, O, LSE)
        dK, _ = oattn.attn_dkv(qr, kr, v, do, wl.cu_seqlens, wl.softmax_scale, rows, O, LSE)
        assert rel(f64(dev_to_bits(ra.o)), O) <= 2e-2
        assert rel(dq, turn(dQ, want, turns, rot, -1)) <= 2e-2 and rel(dk, turn(dK, pos_k, turns, rot, -1)) <= 2e-2
    # the direct way: bf16 gradients turned in place, one rounding more
    ra.forward_direct()
    ra.backward_direct()
    ra.rotate_grads()
    assert rel(f64(dev_to_bits(ra.dq)), dq) <= 2e-2 and rel(f64(dev_to_bits(ra.dk)), dk) <= 2e-2


@pytest.mark.gpu
def test_rotated_pass_in_a_graph():
    import torch
    from paper_2602_21788_amd.rank import RankAttention
    ra = RankAttention([400, 90], [2, 1], 0, 4, 2, 64)
    ra.set_rotary(B.fcp_rotary_frequencies(64)[0])
    ra.set_random_inputs(3)
    q0, k0 = ra.q.clone(), ra.k.clone()

    def step():
        ra.q.copy_(q0), ra.k.copy_(k0)
        ra.rotate_inputs()
        ra.forward_direct()
        ra.backward_direct()
        ra.rotate_grads()

    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        q0.mul_(0.9)
        step()
        eager = [t.clone() for t in (ra.o, ra.dk, ra.dv)]
        dq = ra.dq.float()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (ra.o, ra.dk, ra.dv))), i
        # (dQ of the rows that several items add to: any order)
        assert float((ra.dq.float() - dq).abs().max()) <= 2.0 ** -7 * float(dq.abs().max()), i
