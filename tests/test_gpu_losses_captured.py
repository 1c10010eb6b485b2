"""The losses whose gradient is formed with them (policy, distillation), where only one of the forward
and the backward is captured into a graph, or each into one of its own: every replay gives the gradient
for the factor that it finds, and what a caller holds stays his."""
import pytest

from gpu_util import dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F = pytest.importorskip("paper_2410_15352_amd.functional")
FT = pytest.importorskip("paper_2410_15352_amd.finetune")

ROWS, V, K = 40, 1003, 5


@pytest.fixture(params=["policy", "distill"])
def loss_of(request, monkeypatch):
    for module, name in ((FT, "_policy_torch"), (F, "_distill_torch")):
        monkeypatch.setattr(module, name, None)
    g = torch.Generator(device=dev()).manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=g, device=dev())
    ids = torch.randint(V, (ROWS, K), generator=g, device=dev())
    t = torch.randint(V, (ROWS,), generator=g, device=dev())
    top, old, A = rand(ROWS, K), 0.1 * rand(ROWS) - 7.0, rand(ROWS)
    if request.param == "policy":
        return lambda x: FT.policy_loss(x, t, old, A)[0]
    return lambda x: F.distill_loss(x, top, ids, targets=t, weight=0.5)


def _logits(seed=1):
    g = torch.Generator(device=dev()).manual_seed(seed)
    return torch.randn((ROWS, V), generator=g, device=dev()).to(torch.bfloat16).requires_grad_(True)


def _eager(loss_of, x, factor):
    x = x.detach().requires_grad_(True)
    loss = loss_of(x)
    return torch.autograd.grad(loss, x, torch.full_like(loss, factor))[0]


def _on_a_stream(run):
    """(A capture takes the streams of the nodes that it meets: all are made on this one.)"""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(s)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()


def test_backward_captured_alone(loss_of):
    def run(s):
        x = _logits()
        want = {f: _eager(loss_of, x, f) for f in (1.0, 2.0, -3.0)}
        loss = loss_of(x)
        factor = torch.ones_like(loss)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            (g,) = torch.autograd.grad(loss, x, factor, retain_graph=True)
        for f in (1.0, 2.0, 1.0, -3.0, 1.0, 1.0):
            factor.fill_(f)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(g, want[f])
            g.mul_(0.5)  # (as a clipping in place does)
            assert torch.equal(_eager(loss_of, x, f), want[f])
        (g,) = torch.autograd.grad(loss, x, torch.ones_like(loss))
        assert torch.equal(g, want[1.0])
    _on_a_stream(run)


def test_forward_captured_alone(loss_of):
    def run(s):
        x, other = _logits(), _logits(seed=2)
        first, second = _eager(loss_of, x, 1.0), _eager(loss_of, other, 1.0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            loss = loss_of(x)
        graph.replay()
        (g,) = torch.autograd.grad(loss, x, retain_graph=True)
        assert torch.equal(g, first)
        x.data.copy_(other.detach())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(g, first)  # the caller's own
        (h,) = torch.autograd.grad(loss, x, retain_graph=True)
        assert torch.equal(h, second) and torch.equal(g, first)
    _on_a_stream(run)


def test_forward_and_backward_in_graphs_of_their_own(loss_of):
    x = _logits()
    want = {f: _eager(loss_of, x, f) for f in (1.0, 2.0)}
    graphed = torch.cuda.make_graphed_callables(loss_of, (_logits(seed=2),))
    for _ in range(2):
        loss = graphed(x)
        for f in (1.0, 2.0, 1.0, 1.0):
            (g,) = torch.autograd.grad(loss, x, torch.full_like(loss, f), retain_graph=True)
            torch.cuda.synchronize()
            assert torch.equal(g, want[f])


def test_both_in_one_graph(loss_of):
    """The gradient of the forward's own capture is the one that is given."""
    def run(s):
        x = _logits()
        want = {f: _eager(loss_of, x, f) for f in (1.0, 2.0)}
        factor = torch.ones((), device=dev())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            loss = loss_of(x)
            g, h = (torch.autograd.grad(loss, x, factor, retain_graph=True)[0] for _ in range(2))
        for f in (1.0, 2.0, 1.0, 1.0):
            factor.fill_(f)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(g, want[f]) and torch.equal(h, want[f])
            g.zero_(), h.zero_()
            assert torch.equal(_eager(loss_of, x, f), want[f])
    _on_a_stream(run)
