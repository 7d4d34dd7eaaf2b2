"""Gradients of sekv.rotate through autograd: the formula's, differences, and those of calls in use."""

import pytest
import torch

from tests.rotary_common import bound, frequencies, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _case(S, dtype, layout, n=37, heads=3, dim=64, R=48, scale=1.25, seed=1):
    g = torch.Generator().manual_seed(seed)
    f = frequencies(R)
    x, u = (torch.randn((n, heads, dim), generator=g).to(dtype) for _ in "xu")
    pos = torch.randint(-50, 5000, (n,), generator=g).int()
    return x, u, pos, f, S.Rotary(f.cuda(), layout=layout, scale=scale), scale


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("transpose", [False, True])
def test_gradient(S, dtype, layout, transpose):
    """The result is that of the call without a gradient; the gradient of sum(u y) is u turned the other way, and so are
    differences of the call, which is linear."""
    x, u, pos, f, r, scale = _case(S, dtype, layout)
    leaf = x.cuda().requires_grad_()
    y = S.rotate(leaf, pos.cuda(), r, transpose=transpose)
    with torch.no_grad():
        assert torch.equal(y, S.rotate(leaf, pos.cuda(), r, transpose=transpose))
        assert not S.rotate(leaf, pos.cuda(), r).requires_grad
    assert y.requires_grad
    y.backward(u.cuda())
    want = turned(u, pos, f, layout, scale, not transpose)
    assert leaf.grad.dtype == dtype
    assert ((leaf.grad.cpu().double() - want).abs() <= bound(u, want, dtype, scale)).all()
    if dtype == torch.float32:
        at = y.detach().cpu().double()
        for j in range(0, 64, 9):
            step = x.clone()
            step[..., j] += 1.0
            h = step[..., j].double() - x[..., j].double()
            moved = S.rotate(step.cuda(), pos.cuda(), r, transpose=transpose).cpu().double()
            diff = ((moved - at) * u.double()).sum(-1) / h
            # both results are rounded to float, 2^-24 of each value
            tol = (2.0 ** -24 * 1.01 * (moved.abs() + at.abs()) * u.double().abs()).sum(-1) / h.abs() + 2.0 ** -23 * want[..., j].abs() + 1e-12
            assert ((leaf.grad[..., j].cpu().double() - diff).abs() <= tol).all()


def test_slices_sums_and_unaligned_gradients(S):
    """Heads of a wider projection, an expanded gradient, and one that starts off a 16-byte border."""
    x, _, pos, f, r, scale = _case(S, torch.float32, "half")
    wide = torch.randn((37, 7, 64), device="cuda").requires_grad_()
    S.rotate(wide[:, 2:5], pos.cuda(), r).sum().backward()
    one = torch.ones(37, 3, 64)
    want = turned(one, pos, f, "half", scale, True)
    assert ((wide.grad[:, 2:5].cpu().double() - want).abs() <= bound(one, want, torch.float32, scale)).all()
    assert not wide.grad[:, :2].any() and not wide.grad[:, 5:].any()
    leaf = x.cuda().requires_grad_()
    flat = torch.randn(37 * 3 * 64 + 1, device="cuda")[1:].view(37, 3, 64)
    assert flat.data_ptr() % 16
    S.rotate(leaf, pos.cuda(), r).backward(flat)
    assert torch.equal(leaf.grad, S.rotate(flat.clone(), pos.cuda(), r, transpose=True))
    none = torch.randn((0, 3, 64), device="cuda").requires_grad_()
    S.rotate(none, pos.cuda()[:0], r).sum().backward()
    assert none.grad.shape == (0, 3, 64)


def test_second_gradient(S):
    """Of |turned x|^2 / 2: the turn there and back, scale^2 of the turned part, twice over."""
    x, u, pos, f, r, scale = _case(S, torch.float32, "interleaved")
    leaf = x.cuda().requires_grad_()
    y = S.rotate(leaf, pos.cuda(), r)
    first, = torch.autograd.grad((y * y).sum() / 2, leaf, create_graph=True)
    second, = torch.autograd.grad((first * u.cuda()).sum(), leaf)
    factor = torch.where(torch.arange(64) < 48, scale ** 2, 1.0).double()
    # two turns, each result within its bound
    tol = 2 * scale * (bound(x, x.abs().amax(-1, keepdim=True) * 2 * scale, torch.float32, scale)) + 2.0 ** -22 * x.abs() * scale ** 2
    assert ((first.detach().cpu().double() - factor * x.double()).abs() <= tol).all()
    tol = 2 * scale * (bound(u, u.abs().amax(-1, keepdim=True) * 2 * scale, torch.float32, scale)) + 2.0 ** -22 * u.abs() * scale ** 2
    assert ((second.cpu().double() - factor * u.double()).abs() <= tol).all()


def test_another_stream(S):
    """Forward and backward on a stream that is not the current one, with its inputs late there."""
    x, u, pos, f, r, scale = _case(S, torch.float32, "half", n=4096)
    leaf, p, want = x.cuda().requires_grad_(), pos.cuda(), turned(u, pos, f, "half", scale, True)
    late = torch.zeros(4096, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        a = torch.randn((3000, 3000), device="cuda")
        for _ in range(20):
            a = a @ a / 60.0
        late.copy_(p)
    y = S.rotate(leaf, late, r, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    y.backward(u.cuda())
    assert ((leaf.grad.cpu().double() - want).abs() <= bound(u, want, torch.float32, scale)).all()


def test_changed_positions_are_noticed_and_out_is_refused(S):
    x, u, pos, f, r, _ = _case(S, torch.float32, "half")
    leaf, p = x.cuda().requires_grad_(), pos.cuda()
    y = S.rotate(leaf, p, r)
    p.add_(1)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward(u.cuda())
    for a, out in ((leaf, torch.empty_like(u, device="cuda")), (leaf, leaf), (u.cuda(), leaf)):
        with pytest.raises(ValueError, match="out"):
            S.rotate(a, p, r, out=out)
    with torch.no_grad():
        S.rotate(leaf, p, r, out=leaf)


def test_captured_and_replayed(S):
    """Forward and backward in one graph, replayed with new inputs, eager passes of the same leaf between."""
    x, u, pos, f, r, scale = _case(S, torch.bfloat16, "half")
    leaf, p, up = x.cuda().requires_grad_(), pos.cuda(), u.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(S.rotate(leaf, p, r), leaf, up)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = S.rotate(leaf, p, r)
        grad, = torch.autograd.grad(y, leaf, up)
        y = y.detach()
    g = torch.Generator().manual_seed(9)
    for _ in range(4):
        with torch.no_grad():
            leaf.copy_(torch.randn(x.shape, generator=g))
        up.copy_(torch.randn(u.shape, generator=g))
        p.copy_(torch.randint(0, 9000, p.shape, generator=g).int())
        graph.replay()
        got = y.clone(), grad.clone()
        eager = S.rotate(leaf, p, r)
        want, = torch.autograd.grad(eager, leaf, up)
        torch.cuda.synchronize()
        assert torch.equal(got[0], eager) and torch.equal(got[1], want)
