"""Rotary positions on the GPU against 64 bits."""
from fractions import Fraction
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
F64 = torch.float64
PI = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)


def angles(pos, freq):
    """pos x freq within half a turn, rounded once."""
    rows = []
    for f in freq.tolist():
        turn = Fraction(f) / (2 * PI)
        rows.append([float((p * turn + Fraction(1, 2)) % 1 - Fraction(1, 2)) for p in pos.tolist()])
    return torch.tensor(rows, dtype=F64).T * 2 * math.pi


def reference(x, pos, freq, layout, scale, inverse):
    """The turned values in 64 bits and how far fp32 may be off: the angle by 2^-24 of pi, sine and cosine by 2 steps of 2^-23, three
    roundings of products and the sum, and the result's own to 16 bits."""
    a = angles(pos, freq).to(x.device) * (-1.0 if inverse else 1.0)
    c, s = torch.cos(a)[:, None] * scale, torch.sin(a)[:, None] * scale
    half = freq.numel()
    i = slice(0, half) if layout == "half" else slice(0, 2 * half, 2)
    j = slice(half, 2 * half) if layout == "half" else slice(1, 2 * half, 2)
    x = x.to(F64)
    y, tol = x.clone(), torch.zeros_like(x)
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    tol[..., i] = tol[..., j] = (math.pi + 4 + 4) * 2.0 ** -24 * abs(scale) * (x[..., i].abs() + x[..., j].abs())
    return y, tol


def check(got, x, pos, freq, layout, scale=1.0, inverse=False):
    y, tol = reference(x, pos, freq, layout, scale, inverse)
    dt = got.dtype
    tol = tol + torch.finfo(dt).eps / 2 * (y.abs() + tol) + (2.0 ** -25 if dt == torch.float16 else 0.0)
    rot = 2 * freq.numel()
    assert torch.equal(got[..., rot:], x[..., rot:])
    bad = (got.to(F64) - y).abs()[..., :rot] > tol[..., :rot]
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4], float((got.to(F64) - y).abs().max()))


def make(T, Hq, Hkv, D, dt, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qk = torch.randn(T, Hq + Hkv, D, device="cuda", generator=g).to(dt)
    pos = torch.randint(0, 1 << 20, (T,), device="cuda", generator=g).int()
    return qk[:, :Hq], qk[:, Hq:], pos


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot", [(1, 4, 1, 64, 64), (7, 5, 3, 128, 128), (33, 8, 2, 128, 32), (64, 3, 3, 64, 20), (9, 2, 1, 80, 80),
                                            (5, 1, 1, 8, 2), (40, 2, 2, 512, 512), (13, 7, 1, 256, 48), (1300, 4, 4, 64, 64), (1201, 3, 2, 72, 16)])
def test_turns_by_positions(dt, layout, T, Hq, Hkv, D, rot):
    from paper_2511_01282_gb300 import rotary
    q, k, pos = make(T, Hq, Hkv, D, dt)
    pos[:1], pos[-1:] = 0, -3
    f = rotary.frequencies(rot, 500000.0, 8.0, 8192)
    r = rotary.Rotary(D, rot, layout, f, 1.25)
    for inverse in (False, True):
        a, b = r(q, k, pos, inverse=inverse)
        check(a, q, pos, f, layout, 1.25, inverse)
        check(b, k, pos, f, layout, 1.25, inverse)
    # in place, the same bits
    x = torch.cat([q, k], 1)
    c, d = r(x[:, :Hq], x[:, Hq:], pos, out=(x[:, :Hq], x[:, Hq:]), inverse=True)
    assert torch.equal(x[:, :Hq], a) and torch.equal(x[:, Hq:], b) and c.data_ptr() == x.data_ptr()
    # queries alone, keys alone
    assert torch.equal(r(q, None, pos, inverse=True)[0], a) and torch.equal(r(None, k, pos, inverse=True)[1], b)


def test_far_positions():
    from paper_2511_01282_gb300 import rotary
    q, k, pos = make(64, 2, 1, 64, torch.float16)
    pos[:] = torch.tensor([2 ** 31 - 1 - i for i in range(32)] + [-2 ** 31 + i for i in range(32)], dtype=torch.int32)
    f = rotary.frequencies(64)
    a, b = rotary.Rotary(64)(q, k, pos)
    check(a, q, pos, f, "half")
    check(b, k, pos, f, "half")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_gradient(layout):
    """The inverse call is the gradient: of a sum w.y against differences (the map is linear: exact in 64 bits) and against autograd."""
    from paper_2511_01282_gb300 import rotary
    dt, D, rot = torch.bfloat16, 64, 48
    q, k, pos = make(11, 3, 2, D, dt)
    r = rotary.Rotary(D, rot, layout, scale=0.75)
    w = make(11, 3, 2, D, dt, 2)[0]
    grad, _ = r(w, None, pos, inverse=True)
    x = q.to(F64).requires_grad_()
    y, _ = reference(x, pos, r.freq, layout, 0.75, False)
    (y * w.to(F64)).sum().backward()
    scale = 0.75 * (w.to(F64).abs().amax() * 2)
    assert ((grad.to(F64) - x.grad).abs() <= scale * (2.0 ** -9 + 12 * 2.0 ** -24)).all()
    base = (reference(q, pos, r.freq, layout, 0.75, False)[0] * w.to(F64)).sum()
    for i in ((0, 0, 0), (5, 2, rot - 1), (10, 1, D - 1), (3, 0, 7)):
        step = q.to(F64).clone()
        step[i] += 1.0
        diff = (reference(step, pos, r.freq, layout, 0.75, False)[0] * w.to(F64)).sum() - base
        assert abs(float(grad[i].to(F64) - diff)) <= scale * (2.0 ** -9 + 12 * 2.0 ** -24) + 1e-9


def test_graphs_streams_and_no_rows():
    from paper_2511_01282_gb300 import respec as rs, rotary
    q, k, pos = make(50, 4, 2, 128, torch.bfloat16)
    r = rotary.Rotary(128)
    a, b = r(q, k, pos)
    q2, k2 = torch.zeros_like(a), torch.zeros_like(b)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        r(q, k, pos, out=(q2, k2))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, q2) and torch.equal(b, k2)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c, d = r(q, k, pos)
    side.synchronize()
    assert torch.equal(a, c) and torch.equal(b, d)
    n = rs.rs_launch_count()
    r(q[:0], k[:0], pos[:0])
    assert rs.rs_launch_count() == n


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("inverse", [False, True])
def test_gradients_reach_queries_and_keys(layout, dt, inverse):
    """Through autograd: the bits of the call with the opposite angles, for parts of wider rows, broadcast and transposed gradients,
    for one of the two alone, and twice."""
    from paper_2511_01282_gb300 import rotary
    D, rot, T = 64, 48, 11
    r = rotary.Rotary(D, rot, layout, scale=0.75)
    x = torch.cat(make(T, 3, 2, D, dt)[:2], 1).requires_grad_()
    pos = make(T, 3, 2, D, dt)[2]
    wq, wk, _ = make(T, 3, 2, D, dt, 2)
    a, b = r(x[:, :3], x[:, 3:], pos, inverse=inverse)
    with torch.no_grad():
        c, d = r(x[:, :3], x[:, 3:], pos, inverse=inverse)
        dq, dk = r(wq, wk, pos, inverse=not inverse)
    assert a.requires_grad and b.requires_grad and not c.requires_grad and torch.equal(a, c) and torch.equal(b, d)
    g, = torch.autograd.grad((a, b), x, (wq, wk), retain_graph=True)
    assert torch.equal(g[:, :3], dq) and torch.equal(g[:, 3:], dk)
    g, = torch.autograd.grad(b, x, wk, retain_graph=True)
    assert (g[:, :3] == 0).all() and torch.equal(g[:, 3:], dk)
    # of a sum (one value for all), and with heads and rows the other way round
    g, = torch.autograd.grad(a.sum(), x, retain_graph=True)
    with torch.no_grad():
        assert torch.equal(g[:, :3], r(torch.ones_like(a), None, pos, inverse=not inverse)[0])
    g, = torch.autograd.grad(a.transpose(0, 1), x, wq.transpose(0, 1).contiguous(), retain_graph=True)
    assert torch.equal(g[:, :3], dq)
    # keys alone need one; and the gradient of the gradient, which is linear in what came in
    k = make(T, 3, 2, D, dt)[1].clone().requires_grad_()
    q2, k2 = r(wq, k, pos, inverse=inverse)
    assert k2.requires_grad and not q2.requires_grad
    w = wk.clone().requires_grad_()
    g, = torch.autograd.grad(k2, k, w, create_graph=True)
    gg, = torch.autograd.grad(g, w, wk)
    with torch.no_grad():
        assert torch.equal(gg, r(None, wk, pos, inverse=inverse)[1])


def test_gradients_of_one_side_stream_and_of_no_rows():
    from paper_2511_01282_gb300 import rotary
    q, k, pos = make(50, 4, 2, 128, torch.bfloat16)
    r = rotary.Rotary(128)
    want = r(q, None, pos, inverse=True)[0]
    leaf = torch.zeros_like(q).requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a, _ = r(leaf, None, pos)
        a.backward(q)
    side.synchronize()
    assert torch.equal(leaf.grad, want)
    none = q[:0].clone().requires_grad_()
    a, _ = r(none, None, pos[:0])
    a.sum().backward()
    assert none.grad.shape == (0, 4, 128)
