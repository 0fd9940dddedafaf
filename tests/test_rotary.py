"""Rotary positions against the definition in 64 bits, the adjoint against the definition of an adjoint and against differences, the frequencies
against their formulas, and the refusals (on the CPU)."""
import ctypes
import math

import numpy as np
import pytest

from paper_2602_21788_amd import binding as B

TYPES = {"bf16": "bfloat16", "f32": "float32"}


# ---- CPU ------------------------------------------------------------------------------------------------------------------------------------
def test_frequencies_follow_their_formulas():
    r, base, s, L0 = 64, 10000.0, 8.0, 4096.0
    i = np.arange(r // 2)
    f = base ** (-2.0 * i / r) / (2 * math.pi)
    t, m = B.fcp_rotary_frequencies(r, base)
    assert np.allclose(t, f, rtol=1e-14) and m == 1
    t, m = B.fcp_rotary_frequencies(r, base, B.FCP_ROTARY_LINEAR, s)
    assert np.allclose(t, f / s, rtol=1e-14) and m == 1
    t, m = B.fcp_rotary_frequencies(r, base, B.FCP_ROTARY_BASE, s)
    assert t[0] == f[0] and math.isclose(t[-1], f[-1] / s, rel_tol=1e-12) and m == 1
    t, m = B.fcp_rotary_frequencies(r, base, B.FCP_ROTARY_PARTS, s, L0, 1.0, 32.0)
    turns, plain = L0 * f, B.fcp_rotary_frequencies(r, base)[0]
    assert np.array_equal(t[turns >= 32], plain[turns >= 32]) and np.allclose(t[turns <= 1], f[turns <= 1] / s, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    g = (turns[mid] - 1) / 31
    assert mid.any() and np.allclose(t[mid], g * f[mid] + (1 - g) * f[mid] / s, rtol=1e-13)
    assert math.isclose(m, 0.1 * math.log(s) + 1, rel_tol=1e-6)


def test_frequency_refusals():
    for args in (dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=8, base=0.0), dict(rot_dim=8, base=float("nan")),
                 dict(rot_dim=8, scaling=B.FCP_ROTARY_LINEAR, factor=0.5), dict(rot_dim=2, scaling=B.FCP_ROTARY_BASE, factor=2.0),
                 dict(rot_dim=8, scaling=B.FCP_ROTARY_PARTS, factor=2.0, original_len=0.0),
                 dict(rot_dim=8, scaling=B.FCP_ROTARY_PARTS, factor=2.0, original_len=10.0, low=4.0, high=4.0)):
        with pytest.raises(B.FcpError) as e:
            B.fcp_rotary_frequencies(**args)
        assert e.value.code == B.FCP_ERR_INVALID_ARG
    with pytest.raises(B.FcpError) as e:
        B.fcp_rotary_frequencies(8, scaling=7)
    assert e.value.code == B.FCP_ERR_UNSUPPORTED


def test_rotary_refusals_come_before_any_device_work():
    L = B.lib()
    fake = 0x10000                                # never dereferenced: every call fails first, or has nothing to do

    def call(n=1, dim=128, rot=128, layout=0, magnitude=1.0, backward=0, turns=fake, **kw):
        p = (B.RotaryPart * max(n, 1))()
        for a in p:
            a.x = a.y = a.pos = fake
            a.x_row = a.y_row = 4 * 128
            a.x_head = a.y_head = 128
            a.rows, a.heads = 5, 4
            for name, v in kw.items():
                setattr(a, name, v)
        return L.fcp_rotary(p, n, turns, dim, rot, layout, magnitude, backward, None)

    bad, no = B.FCP_ERR_INVALID_ARG, B.FCP_ERR_UNSUPPORTED
    assert call(n=-1) == bad and call(turns=None) == bad and L.fcp_rotary(None, 1, fake, 128, 128, 0, 1.0, 0, None) == bad
    assert call(n=5) == no and b"at most 4" in L.fcp_last_error()
    assert call(dim=1) == no and call(dim=1026) == no
    assert call(rot=3) == bad and call(rot=130) == bad and call(rot=0) == bad
    assert call(layout=2) == bad and call(backward=2) == bad and call(magnitude=0.0) == bad and call(magnitude=float("inf")) == bad
    assert call(rows=-1) == bad and call(heads=-1) == bad and call(x=None) == bad and call(pos=None) == bad
    assert call(x_type=2) == no and call(y_type=-1) == no
    assert call(x_row=-1) == bad and call(y_row=64) == bad and call(y_head=64) == bad
    assert call(y_type=B.FCP_F32) == bad and b"in place" in L.fcp_last_error()
    assert call(x=fake + 1, y=fake + 1) == bad and b"aligned" in L.fcp_last_error()
    assert call(n=0) == 0 and call(rows=0) == 0 and call(heads=0, x=None) == 0


# ---- GPU ------------------------------------------------------------------------------------------------------------------------------------
def reference(x, pos, turns, rot, half, magnitude, backward):
    """(y, bound of the error before the last rounding) in 64 bits.  The fraction of a turn as a float: off by 2^-26 turns, 9.4e-8 rad; cosine and sine by 2 units of
    2^-23; two products and a sum by 3 * 2^-24: at most 6e-7 of |a| + |b|."""
    t = pos.astype(np.float64)[:, None] * turns
    a = 2 * math.pi * (t - np.rint(t)) * (-1 if backward else 1)
    c, s = np.cos(a)[:, None] * magnitude, np.sin(a)[:, None] * magnitude
    ia = np.arange(rot // 2) if half else 2 * np.arange(rot // 2)
    ib = ia + rot // 2 if half else ia + 1
    y, err = x.copy(), np.zeros_like(x)
    xa, xb = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = xa * c - xb * s, xa * s + xb * c
    err[..., ia] = err[..., ib] = 6e-7 * magnitude * (np.abs(xa) + np.abs(xb))
    return y, err


def check(y, x, *args, dtype):
    import torch
    want, err = reference(x.double().cpu().numpy(), *args)
    got = y.double().cpu().numpy()
    tol = err + np.abs(want) * (torch.finfo(dtype).eps / 2) + 1e-38
    assert (np.abs(got - want) <= tol * (1 + 1e-3)).all(), float((np.abs(got - want) / tol).max())


@pytest.mark.gpu
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("rows,heads,dim,rot,x_type,y_type", [
    (1, 1, 64, 64, "bf16", "bf16"), (1, 32, 128, 128, "bf16", "bf16"), (17, 8, 128, 32, "bf16", "bf16"), (300, 40, 128, 128, "f32", "bf16"),
    (61, 6, 64, 48, "f32", "f32"), (7, 3, 72, 20, "bf16", "f32"), (5, 2, 96, 96, "bf16", "bf16"), (1031, 5, 128, 64, "bf16", "bf16"),
    (3, 2, 10, 2, "f32", "bf16"), (2, 2, 1024, 1024, "f32", "f32"), (4, 1, 1022, 1022, "bf16", "bf16"), (4099, 10, 64, 64, "bf16", "bf16")])
def test_rotary_matches_the_definition(rows, heads, dim, rot, x_type, y_type, half, backward):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + dim)
    xt, yt = getattr(torch, TYPES[x_type]), getattr(torch, TYPES[y_type])
    x = torch.randn(rows, heads, dim, generator=g, device="cuda").to(xt)
    y = torch.full((rows, heads, dim), float("nan"), dtype=yt, device="cuda")
    pos = torch.randint(-5, 1 << 20, (rows,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = 0 if rows > 1 else (1 << 31) - 1
    turns, m = B.fcp_rotary_frequencies(rot, 500000.0, B.FCP_ROTARY_PARTS if rot > 2 else B.FCP_ROTARY_PLAIN, 4.0, 8192.0)
    B.fcp_rotary([(x, y, pos)], torch.from_numpy(turns).cuda(), rot, B.FCP_ROTARY_HALF if half else B.FCP_ROTARY_PAIRS, m, backward)
    check(y, x, pos.cpu().numpy(), turns, rot, half, m, backward, dtype=yt)


@pytest.mark.gpu
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("offset", [0, 8, 3])
def test_rotary_of_strided_rows_in_place_and_beside_others(half, offset):
    """Queries and keys of a fused projection, in place, two tensors in a launch, nothing else of the buffer touched."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    n, hq, hkv, D = 37, 6, 2, 64
    buf = torch.randn(n, (hq + 2 * hkv) * D + 16, generator=g, device="cuda").to(torch.bfloat16)
    before = buf.clone()
    row = buf[:, offset: offset + (hq + 2 * hkv) * D].unflatten(1, (-1, D))
    q, k = row[:, :hq], row[:, hq: hq + hkv]
    q0, k0 = q.clone(), k.clone()
    pos = torch.randint(0, 131072, (n,), generator=g, device="cuda", dtype=torch.int32)
    turns, _ = B.fcp_rotary_frequencies(D)
    td = torch.from_numpy(turns).cuda()
    layout = B.FCP_ROTARY_HALF if half else B.FCP_ROTARY_PAIRS
    B.fcp_rotary([(q, q, pos), (k, k, pos)], td, D, layout)
    for y, x in ((q, q0), (k, k0)):
        check(y, x, pos.cpu().numpy(), turns, D, half, 1.0, False, dtype=torch.bfloat16)
    q.copy_(q0), k.copy_(k0)
    assert torch.equal(buf.view(torch.int16), before.view(torch.int16))


@pytest.mark.gpu
def test_rotary_of_heads_first_and_broadcast_inputs():
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(4, 29, 64, generator=g, device="cuda").to(torch.bfloat16).transpose(0, 1)          # [rows, heads, D], heads outermost
    y = torch.empty(4, 29, 64, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    pos = torch.arange(29, device="cuda", dtype=torch.int32)
    turns, _ = B.fcp_rotary_frequencies(64)
    B.fcp_rotary([(x, y, pos)], torch.from_numpy(turns).cuda(), 64)
    check(y, x, pos.cpu().numpy(), turns, 64, True, 1.0, False, dtype=torch.bfloat16)
    one = torch.randn(29, 1, 64, generator=g, device="cuda").to(torch.bfloat16).expand(29, 4, 64)
    z = torch.empty(29, 4, 64, device="cuda", dtype=torch.bfloat16)
    B.fcp_rotary([(one, z, pos)], torch.from_numpy(turns).cuda(), 64)
    check(z, one, pos.cpu().numpy(), turns, 64, True, 1.0, False, dtype=torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("half", [True, False])
def test_backward_is_the_adjoint_and_agrees_with_differences(half):
    """In fp32: <R x, w> = <x, R' w>; and the derivative of <R x, w> by an element of x, by a central difference, is that element of R' w.  R is linear, so the difference
    has no error of its own, only rounding: 2 h = 1, each of D terms off by at most 1e-6 |x| |w|."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    n, h, D, rot = 9, 2, 64, 32
    mk = lambda: torch.randn(n, h, D, generator=g, device="cuda")
    x, w = mk(), mk()
    pos = torch.randint(0, 100000, (n,), generator=g, device="cuda", dtype=torch.int32)
    turns = torch.from_numpy(B.fcp_rotary_frequencies(rot)[0]).cuda()
    layout = B.FCP_ROTARY_HALF if half else B.FCP_ROTARY_PAIRS

    def turn(v, backward=False):
        y = torch.empty_like(v)
        B.fcp_rotary([(v, y, pos)], turns, rot, layout, 1.3, backward)
        return y.double()

    back = turn(w, True)
    assert abs(float((turn(x) * w.double()).sum() - (x.double() * back).sum())) <= 1e-6 * float((x.abs() * w.abs()).double().sum()) * 4
    for at in ((0, 0, 0), (4, 1, 5), (8, 0, 17), (3, 1, 31), (2, 1, 40)):
        up, down = x.clone(), x.clone()
        up[at] += 0.5
        down[at] -= 0.5
        diff = ((turn(up) - turn(down)) * w.double()).sum() / float(up[at].double() - down[at].double())
        assert abs(float(diff) - float(back[at])) <= 1e-5 * 4


@pytest.mark.gpu
def test_rotary_on_another_stream_and_in_a_graph():
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(64, 8, 128, generator=g, device="cuda").to(torch.bfloat16)
    y, z = torch.empty_like(x), torch.empty_like(x)
    pos = torch.randint(0, 4096, (64,), generator=g, device="cuda", dtype=torch.int32)
    turns = torch.from_numpy(B.fcp_rotary_frequencies(128)[0]).cuda()
    B.fcp_rotary([(x, y, pos)], turns, 128)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        B.fcp_rotary([(x, z, pos)], turns, 128)
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    with torch.cuda.graph(graph):
        B.fcp_rotary([(x, z, pos)], turns, 128)
    for i in range(3):
        x.copy_(torch.randn(64, 8, 128, generator=g, device="cuda"))
        pos.add_(1000)
        graph.replay()
        B.fcp_rotary([(x, y, pos)], turns, 128)
        torch.cuda.synchronize()
        assert torch.equal(y, z), i
