"""rope in a program that trains: its graph, the gradient against the formula in 64
bits and against differences, twice, through broadcast and strided gradients, in a
captured step; what it refuses where a gradient would be lost."""
import pytest
import torch

from test_rope_append import check_turned, frequencies, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_09721_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "no GPU"
    return binding


def inputs(shape, dtype, axes=1, seed=1, pairs=None):
    g = torch.Generator().manual_seed(seed)
    n = 1
    for s in shape[:-2]:
        n *= s
    x = torch.randn(shape, generator=g).to(dtype).cuda()
    inv, axis = frequencies(pairs or shape[-1] // 2, axes, g)
    pos = torch.randint(-50000, 50000, (axes, n), generator=g).int().cuda()
    return x, pos, inv, axis, torch.randn(shape, generator=g).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape,axes,pairs", [((7, 3, 64), 1, 32), ((130, 4, 128), 3, 32), ((2, 9, 2, 64), 1, 16), ((1, 1, 64), 1, 32)])
def test_gradient(B, shape, axes, pairs, interleaved, dtype):
    x, pos, inv, axis, dy = inputs(shape, dtype, axes, pairs=pairs)
    leaf = x.clone().requires_grad_()
    y = B.rope(leaf, pos, inv, axis, interleaved)
    assert y.requires_grad and torch.equal(y.detach(), B.rope(x, pos, inv, axis, interleaved))
    y.backward(dy)
    rows = lambda t: t.reshape(-1, *shape[-2:])
    check_turned(rows(leaf.grad), rows(dy), pos, inv, axis, interleaved, True)
    assert torch.equal(leaf.grad, B.rope_bwd(dy, pos, inv, axis, interleaved))


def test_gradient_by_differences(B):
    """d/dh loss(x + h e) at 0 of loss = sum w rope(x)^3, by central differences in 64 bits of the oracle."""
    x, pos, inv, axis, w = inputs((20, 3, 64), torch.float32, 3)
    leaf = x.clone().requires_grad_()
    (B.rope(leaf, pos, inv, axis).pow(3) * w).sum().backward()
    e = torch.randn(x.shape, generator=torch.Generator().manual_seed(2)).double()
    f = lambda t: float((turned(t, pos, inv, axis, False)[0].pow(3) * w.cpu().double()).sum())
    h = 1e-4
    left = (f(x.cpu().double() + h * e) - f(x.cpu().double() - h * e)) / (2 * h)
    right = float((leaf.grad.double().cpu() * e).sum())
    # fp32: 3840 products |e| 3 w y^2 of order 10 at most on average, each off by about 20 2^-24; differences: h^2 of 6 w e^3
    assert abs(left - right) <= 3840 * 10 * 20 * 2.0 ** -24 + 3840 * 20 * h * h and abs(left) > 1


def test_twice(B):
    """The gradient's own gradient: rope is linear, so it is rope."""
    x, pos, inv, axis, dy = inputs((11, 2, 64), torch.float32)
    x, dy = x.requires_grad_(), dy.requires_grad_()
    (g,) = torch.autograd.grad(B.rope(x, pos, inv), x, dy, create_graph=True)
    v = torch.randn_like(g)
    (gg,) = torch.autograd.grad(g, dy, v)
    assert torch.equal(gg, B.rope(v, pos, inv))


def test_broadcast_and_strided_gradients(B):
    x, pos, inv, axis, _ = inputs((2, 6, 4, 64), torch.bfloat16)
    leaf = x.clone().requires_grad_()
    B.rope(leaf, pos, inv).sum().backward()                                   # one value for all
    assert torch.equal(leaf.grad, B.rope_bwd(torch.ones_like(x), pos, inv))
    leaf.grad = None
    y = B.rope(leaf, pos, inv)
    dy = torch.randn(2, 4, 6, 64, device="cuda").bfloat16()
    y.transpose(1, 2).backward(dy)                                            # heads outside
    assert torch.equal(leaf.grad, B.rope_bwd(dy.transpose(1, 2).contiguous(), pos, inv))
    odd = torch.empty(x.numel() + 1, device="cuda", dtype=x.dtype)[1:].view(x.shape).copy_(dy.transpose(1, 2))
    leaf.grad = None
    B.rope(leaf, pos, inv).backward(odd)                                      # not aligned
    assert torch.equal(leaf.grad, B.rope_bwd(dy.transpose(1, 2).contiguous(), pos, inv))
    full = torch.randn(12, 6, 64, device="cuda").bfloat16().requires_grad_()  # queries of a fused projection
    B.rope(full[:, :4], pos, inv).backward(dy.transpose(1, 2).flatten(0, 1))
    assert torch.equal(full.grad[:, :4], leaf.grad.flatten(0, 1)) and not bool(full.grad[:, 4:].any())


def test_refused_where_a_gradient_would_be_lost(B):
    x, pos, inv, axis, dy = inputs((5, 2, 64), torch.float32)
    leaf = x.clone().requires_grad_()
    for f in (lambda: B.rope(leaf, pos, inv, out=torch.empty_like(x)), lambda: B.rope(leaf * 1, pos, inv, out=x),
              lambda: B.rope(x, pos, inv.clone().requires_grad_())):
        with pytest.raises(ValueError):
            f()
    with torch.no_grad():
        out = torch.empty_like(x)
        assert B.rope(leaf, pos, inv, out=out) is out and torch.equal(out, B.rope(x, pos, inv))
    with torch.inference_mode():
        y = B.rope(x, pos, inv)
        assert not y.requires_grad and B.rope(y, pos, inv, out=y) is y
    # values that a graph still needs, or positions, changed in place: torch's own error
    z = x.clone()
    loss = (leaf * z).sum()
    B.rope(z, pos, inv, out=z)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        loss.backward()
    y = B.rope(leaf, pos, inv)
    pos += 1
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.sum().backward()


def test_captured_training_step(B):
    """Forward and gradient captured together; replays take the inputs as they are by then."""
    x, pos, inv, axis, dy = inputs((33, 2, 128), torch.bfloat16, 3)
    leaf = x.clone().requires_grad_()

    def step():
        (g,) = torch.autograd.grad(B.rope(leaf, pos, inv, axis, True), leaf, dy)
        return g

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        dy.copy_(torch.randn(dy.shape))
        pos.add_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, B.rope_bwd(dy, pos, inv, axis, True)), i
