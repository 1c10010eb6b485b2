"""Rotary positions, windowed attention and distillation on the GPU where a call is unusual:
first under a capture, of very many or very few rows, with keys of infinities."""
import math

import pytest

from gpu_util import dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F = pytest.importorskip("paper_2410_15352_amd.functional")


def _rand(*shape, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device=dev()).manual_seed(seed + sum(shape))
    return torch.randn(*shape, generator=g, device=dev()).to(dtype)


def test_rotary_first_called_under_capture():
    """The frequencies are formed in the graph then, and again by the first call outside it."""
    q = _rand(2, 9, 2, 64)
    ref = F.Rotary(32, scaling="ntk", factor=2.0)(q)
    rope = F.Rotary(32, scaling="ntk", factor=2.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = rope(q)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref)
        assert torch.equal(rope(q), ref)


def test_rotary_first_called_under_a_transform():
    q = _rand(2, 9, 2, 64, dtype=torch.float32)
    rope = F.Rotary(64)
    g = torch.func.grad(lambda x: rope(x).square().sum())(q)
    assert torch.equal(rope(q), F.Rotary(64)(q))
    # of a rotation: |R x|^2 = |x|^2, to fp32's roundings of some products
    assert (g - 2 * q).abs().max() <= 2.0 ** -19 * q.abs().max()


@pytest.mark.parametrize("pair", [False, True])
def test_rotary_positions_written_before_the_backward(pair):
    rope, q, pos = F.Rotary(64), _rand(2, 9, 2, 64).requires_grad_(), torch.arange(9, device=dev())
    y = rope(q, q if pair else None, positions=pos)
    y = y[1] if pair else y
    torch.autograd.grad(y, q, y.detach(), retain_graph=True)
    pos += 9
    with pytest.raises(RuntimeError, match="inplace operation"):
        torch.autograd.grad(y, q, y.detach())
