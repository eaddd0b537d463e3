"""Rotary positions against their definition in 64 bits."""
import math

import pytest

from paper_2608_26004_gb300 import asymspec as A
from paper_2608_26004_gb300 import serving as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as _torch
    assert _torch.cuda.is_available(), "the gpu tests need a CUDA device"
    from paper_2608_26004_gb300 import build
    build.build_cuda()
    S.lib()
    return _torch


def turned(torch, x, positions, rotary, transpose=False):
    """(result, sum of the magnitudes that enter each element) in 64 bits, from the steps as they are."""
    rot = rotary.rotary_dim
    steps = [s + (1 << 64) if s < 0 else s for s in rotary.steps.tolist()]
    # the phase as a whole number; its fraction of a turn in 64 bits
    angle = torch.tensor([[(s * max(p, 0) % (1 << 64)) / 2.0 ** 64 for s in steps] for p in positions.tolist()],
                         dtype=torch.float64) * (2 * math.pi)
    c, s = angle.cos()[:, None] * rotary.magnitude, angle.sin()[:, None] * rotary.magnitude
    if transpose:
        s = -s
    y = x.double().cpu().clone()
    mag = y.abs()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if rotary.interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
    live = (positions.cpu() >= 0)[:, None, None]
    a2, b2 = torch.where(live, c * a - s * b, a), torch.where(live, s * a + c * b, b)
    size = torch.where(live, (a.abs() + b.abs()) * abs(rotary.magnitude), torch.zeros_like(a))
    if rotary.interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = a2, b2
        mag[..., 0:rot:2] = mag[..., 1:rot:2] = size
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = a2, b2
        mag[..., :rot // 2] = mag[..., rot // 2:rot] = size
    mag[..., rot:] = 0.0
    return y, mag


def check(torch, got, x, positions, rotary, transpose=False):
    """Tolerance, of the magnitudes that enter: an angle within an eighth of a turn is rounded by 2^-28
    turns, 2^-25; sine and cosine by two units of 2^-24, times the magnitude 2^-24, and two products and
    a sum 2^-24 each: 2^-21 in all.  Then one rounding of the type, so the bounds are rounded."""
    y, mag = turned(torch, x, positions, rotary, transpose)
    tol = 2.0 ** -21 * mag
    least, most = ((y + t).to(x.dtype).double() for t in (-tol, tol))
    z = got.double().cpu()
    bad = ~((least <= z) & (z <= most))
    assert not bad.any(), (bad.sum(), z[bad][:5], y[bad][:5])


CASES = [
    # T, heads, kv heads, D, rot, interleaved, dtype
    (1, 1, 1, 64, 64, False, "bfloat16"),
    (1, 4, 1, 2, 2, True, "float32"),
    (5, 16, 8, 128, 128, False, "bfloat16"),
    (37, 3, 1, 80, 20, False, "bfloat16"),      # halves off the vectors' boundaries
    (37, 3, 2, 80, 20, True, "bfloat16"),
    (64, 8, 2, 96, 64, True, "float32"),
    (33, 8, 2, 96, 48, False, "float32"),
    (700, 2, 2, 128, 32, False, "bfloat16"),    # several tokens a CTA
    (1000, 32, 8, 64, 64, True, "bfloat16"),
    (3, 200, 50, 256, 256, False, "float32"),   # more heads than a CTA's units
    (2, 5, 3, 1024, 1024, False, "bfloat16"),
    (19, 7, 5, 33, 10, True, "float32"),        # heads of an odd size
    (301, 1, 1, 16, 6, False, "bfloat16"),
]


def inputs(torch, T, h, hk, D, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn(T, (h + 2 * hk) * D, generator=g, device="cuda").to(getattr(torch, dtype))
    q, k = qkv[:, :h * D].unflatten(-1, (h, D)), qkv[:, h * D:(h + hk) * D].unflatten(-1, (hk, D))
    p = torch.randint(0, 2000, (T,), generator=g, device="cuda", dtype=torch.int32)
    special = torch.tensor([-1, 0, 1, 2 ** 31 - 1, 131071, -2 ** 31, 1000003][:T], device="cuda", dtype=torch.int32)
    if T > 1:
        p[:special.numel()] = special
    return q, k, p


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(torch, case, transpose):
    T, h, hk, D, rot, inter, dtype = CASES[case]
    q, k, p = inputs(torch, T, h, hk, D, dtype, 50 + case)
    rotary = S.Rotary(D, rotary_dim=rot, interleaved=inter, scaling=dict(kind="linear", factor=3.0))
    a, b = rotary(q, p, k, transpose=transpose)
    check(torch, a, q, p, rotary, transpose)
    check(torch, b, k, p, rotary, transpose)
    gone = p < 0
    assert torch.equal(a[gone], q[gone]) and torch.equal(a[..., rot:], q[..., rot:])
    # in place, in the projection's own rows: the same bits, and nothing else
    whole = torch.cat([q.flatten(1), k.flatten(1), k.flatten(1)], 1)
    before = whole.clone()
    q2, k2 = whole[:, :h * D].unflatten(-1, (h, D)), whole[:, h * D:(h + hk) * D].unflatten(-1, (hk, D))
    r = rotary(q2, p, k2, transpose=transpose, q_out=q2, k_out=k2)
    assert r[0] is q2 and torch.equal(q2, a) and torch.equal(k2, b)
    assert torch.equal(whole[:, (h + hk) * D:], before[:, (h + hk) * D:])
    # queries alone
    alone, none = rotary(q, p, transpose=transpose)
    assert none is None and torch.equal(alone, a)


@pytest.mark.parametrize("off", [1, 4])
@pytest.mark.parametrize("inter", [False, True])
def test_strides_and_alignments(torch, off, inter):
    """The same bits off the 16-byte boundaries, in rows apart, heads before tokens, and nothing beside."""
    T, h, D = 21, 6, 64
    q, k, p = inputs(torch, T, h, 2, D, "bfloat16", 3)
    rotary = S.Rotary(D, rotary_dim=32, interleaved=inter)
    want, _ = rotary(q, p)
    room = torch.zeros(h * T * (D + off) + off, device="cuda", dtype=torch.bfloat16)
    x = room[off:].view(h, T, D + off)[..., :D].transpose(0, 1)
    x.copy_(q)
    out = torch.zeros_like(room)
    y = out[off:].view(h, T, D + off)[..., :D].transpose(0, 1)
    rotary(x, p, q_out=y)
    assert torch.equal(y, want)
    assert (out[:off] == 0).all() and (out[off:].view(h, T, D + off)[..., D:] == 0).all()
    wide = q[:1].expand(T, h, D)                        # one token's heads under every position
    check(torch, rotary(wide, p)[0], wide, p, rotary)


def test_gradient(torch):
    """The transpose is the gradient: against autograd of the definition, and against differences of a
    scalar of the results.  Rotation is linear, so a central difference is exact but for fp32: outputs are off
    by 2^-21 of the magnitudes that enter, their scalar by the sum, divided by the step."""
    T, h, D, rot = 6, 3, 32, 24
    for inter in (False, True):
        for scaling in (None, dict(kind="ramp", factor=4.0, original_length=64, fast=4.0, slow=0.5)):
            q, k, p = inputs(torch, T, h, 2, D, "float32", 8)
            p = torch.arange(T, device="cuda", dtype=torch.int32) * 7 - 1
            rotary = S.Rotary(D, rotary_dim=rot, interleaved=inter, scaling=scaling)
            g = torch.randn(T, h, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))
            got, _ = rotary(g, p, transpose=True)
            x = q.double().cpu().requires_grad_()
            angle = p.double().cpu()[:, None] * torch.tensor(
                [(s + (1 << 64) if s < 0 else s) / 2.0 ** 64 for s in rotary.steps.tolist()], dtype=torch.float64)
            c, s = ((f(2 * math.pi * angle) * rotary.magnitude)[:, None] for f in (torch.cos, torch.sin))
            a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
            pair = (c * a - s * b, s * a + c * b)
            y = torch.stack(pair, -1).flatten(-2) if inter else torch.cat(pair, -1)
            y = torch.where((p.cpu() >= 0)[:, None, None], torch.cat([y, x[..., rot:]], -1), x)
            (y * g.double().cpu()).sum().backward()
            _, mag = turned(torch, g, p, rotary, True)
            assert ((got.double().cpu() - x.grad).abs() <= 2.0 ** -21 * mag + 2.0 ** -40).all()
            for t, head, d in ((1, 0, 0), (2, 1, rot - 1), (3, 2, rot), (5, 0, 5), (0, 1, 2)):
                step = torch.zeros_like(q)
                step[t, head, d] = 1.0
                up, down = (rotary(q + e * step, p)[0].double() for e in (1.0, -1.0))
                slope = float(((up - down) * g.double()).sum()) / 2
                size = float(((q.abs() + 1).sum(-1)[t, head] * g.abs().amax()) * 2) * abs(rotary.magnitude)
                assert abs(slope - float(got[t, head, d])) <= 2.0 ** -20 * size


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("transpose", [False, True])
def test_autograd(torch, dtype, transpose):
    """Autograd's gradients are the other direction's results, bit for bit: of both, of one alone, of one number for
    all elements, of the gradient itself, and in a graph."""
    T, h, hk, D = 37, 6, 2, 96
    kind = getattr(torch, dtype)
    q, k, p = inputs(torch, T, h, hk, D, dtype, 21)
    gen = torch.Generator(device="cuda").manual_seed(22)
    gq, gk = (torch.randn(x.shape, device="cuda", generator=gen).to(kind) for x in (q, k))
    rotary = S.Rotary(D, rotary_dim=64, scaling=dict(kind="ramp", factor=4.0, original_length=64, fast=4.0, slow=0.5))
    plain = rotary(q, p, k, transpose=transpose)
    want = rotary(gq, p, gk, transpose=not transpose)
    a, b = q.clone().requires_grad_(), k.clone().requires_grad_()
    y, z = rotary(a, p, b, transpose=transpose)
    assert torch.equal(y, plain[0]) and torch.equal(z, plain[1])
    got = torch.autograd.grad((y, z), (a, b), (gq, gk), retain_graph=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(torch.autograd.grad(z, b, gk, retain_graph=True)[0], want[1])
    assert torch.equal(torch.autograd.grad(y, a, gq, retain_graph=True)[0], want[0])
    one, = torch.autograd.grad(y.sum(), a)
    assert torch.equal(one, rotary(torch.ones_like(q), p, transpose=not transpose)[0])
    y, none = rotary(a, p, transpose=transpose)
    assert none is None and torch.equal(torch.autograd.grad(y, a, gq)[0], want[0])
    y, z = rotary(a, p, k, transpose=transpose)          # k needs none
    assert torch.equal(torch.autograd.grad((y, z), a, (gq, gk))[0], want[0])
    # the gradient is linear in what it is given: its own gradient turns again
    c = gq.clone().requires_grad_()
    y, _ = rotary(a, p, transpose=transpose)
    first, = torch.autograd.grad(y, a, c, create_graph=True)
    assert torch.equal(torch.autograd.grad(first, c, q)[0], plain[0])
    # through a projection, leaves accumulate
    w = torch.randn(D, D, device="cuda", generator=gen).to(kind).requires_grad_()
    (rotary((q @ w).contiguous(), p, transpose=transpose)[0] * gq).sum().backward()
    back = (q.flatten(0, 1).mT.double() @ want[0].flatten(0, 1).double())
    size = q.flatten(0, 1).mT.double().abs() @ want[0].flatten(0, 1).double().abs()
    # sums of T * h products, in 32 bits, and one rounding
    assert ((w.grad.double() - back).abs() <= size * (T * h * 2.0 ** -24) + back.abs() * torch.finfo(kind).eps).all()
    with torch.no_grad():
        assert rotary(a, p)[0].grad_fn is None
    with pytest.raises(ValueError):
        rotary(a, p, q_out=torch.empty_like(q))
    p2 = p.clone()
    y, _ = rotary(a, p2, transpose=transpose)
    p2.add_(1)                                          # what the backward pass needs has changed
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y, a, gq)


def test_autograd_in_a_graph_and_on_a_stream(torch):
    q, k, p = inputs(torch, 40, 8, 2, 128, "bfloat16", 23)
    rotary = S.Rotary(128)
    gq = torch.ones_like(q).mul_(0.5)
    want, _ = rotary(gq, p, transpose=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a = q.clone().requires_grad_()
        got, = torch.autograd.grad(rotary(a, p)[0], a, gq)
        s.synchronize()
        assert torch.equal(got, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got, = torch.autograd.grad(rotary(a, p)[0], a, gq)
    p.add_(5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, rotary(gq, p, transpose=True)[0])


def test_there_and_back_and_moved(torch):
    """Turned by p and back is the input but for two results' roundings; turned by p, then by r, it is turned by
    p + r."""
    q, _, _ = inputs(torch, 50, 4, 1, 128, "float32", 11)
    p = torch.arange(50, device="cuda", dtype=torch.int32) * 2003
    rotary = S.Rotary(128)
    there, _ = rotary(q, p)
    back, _ = rotary(there, p, transpose=True)
    half = q[..., :64].abs() + q[..., 64:].abs()
    tol = 2.0 ** -19 * torch.cat([half, half], -1)
    assert ((back - q).abs() <= tol).all()
    moved, _ = rotary(there, torch.full_like(p, 77))
    assert ((moved - rotary(q, p + 77)[0]).abs() <= tol).all()


def test_far_positions_keep_their_angles(torch):
    """The product of two turned vectors depends on the distance of their positions alone, wherever they are."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(1, 2, 64, generator=g, device="cuda")
    rotary = S.Rotary(64, base=500000.0)
    at = lambda n: rotary(x, torch.tensor([n], device="cuda", dtype=torch.int32))[0].double()  # noqa: E731
    near = (at(19)[0, 0] * at(4)[0, 1]).sum()
    size = (x[0, 0].abs().sum() * x[0, 1].abs().amax() * 2).double()
    for n in (10 ** 4, 10 ** 6, 2 ** 31 - 16):
        assert abs((at(n + 15)[0, 0] * at(n)[0, 1]).sum() - near) <= 2.0 ** -19 * size


def test_nan_and_infinity_stay_in_their_pairs(torch):
    q, _, _ = inputs(torch, 9, 2, 1, 64, "bfloat16", 12)
    q = q.clone()
    q[4, 1, 3], q[5, 0, 40] = math.nan, math.inf
    p = torch.full((9,), 5, device="cuda", dtype=torch.int32)
    p[5] = -1
    out, _ = S.Rotary(64, rotary_dim=32)(q, p)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[4, 1, 3] = bad[4, 1, 19] = True
    assert out[bad].isnan().all() and out[5, 0, 40] == math.inf
    bad[5, 0, 40] = True
    assert out[~bad].isfinite().all()


def test_no_tokens_streams_and_a_graph(torch):
    q, k, p = inputs(torch, 40, 8, 2, 128, "bfloat16", 13)
    rotary = S.Rotary(128)
    a, b = rotary(q[:0], p[:0], k[:0])
    assert a.shape == (0, 8, 128) and b.shape == (0, 2, 128)
    want = rotary(q, p, k)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = rotary(q, p, k)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out = [torch.zeros_like(x) for x in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rotary(q, p, k, q_out=out[0], k_out=out[1])
    p.add_(3)
    g.replay()
    torch.cuda.synchronize()
    check(torch, out[0], q, p, rotary)
    check(torch, out[1], k, p, rotary)


def test_refusals(torch):
    q, k, p = inputs(torch, 8, 4, 2, 64, "bfloat16", 14)
    rotary = S.Rotary(64)
    with pytest.raises(ValueError):
        S.Rotary(64, rotary_dim=66)
    with pytest.raises(A.AsymSpecError):
        S.Rotary(64, rotary_dim=7)
    with pytest.raises(A.AsymSpecError):
        rotary(q, p, q_out=torch.zeros(8, 1, 64, device="cuda", dtype=torch.bfloat16).expand(8, 4, 64))
    same = torch.zeros(8, 4, 64, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(A.AsymSpecError):
        rotary(q, p, q, q_out=same, k_out=same)
    with pytest.raises(ValueError):
        rotary(q.cpu(), p, k)
