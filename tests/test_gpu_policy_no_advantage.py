"""Rows of the policy loss whose advantage is zero: no part but the KL term's, however far the ratio is off."""
import math

import pytest

from gpu_util import dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
FT = pytest.importorskip("paper_2410_15352_amd.finetune")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [100, 8201, 70001])
@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_of_no_advantage(monkeypatch, dtype, V, kl):
    monkeypatch.setattr(FT, "_policy_torch", None)
    g = torch.Generator(device=dev()).manual_seed(V)
    x = torch.randn((12, V), generator=g, device=dev()).to(dtype).requires_grad_(True)
    t = torch.randint(V, (12,), generator=g, device=dev())
    t[5] = -100
    old = FT.token_logprobs(x.detach(), t)
    A, ref = torch.randn(12, generator=g, device=dev()), old - 0.3
    A[1] = A[2] = A[3] = 0.0
    A[3] = -A[3]

    def run(old):
        loss, logp = FT.policy_loss(x, t, old, A, reference=ref, kl=kl)
        g, _ = (torch.autograd.grad(loss, x, retain_graph=True)[0] for _ in range(2))
        h = torch.autograd.grad(FT.policy_loss(x, t, old, A, reference=ref, kl=kl)[0] * 2, x)[0]
        return loss, logp, g, h

    want = run(old)
    for far in (-1000.0, 1000.0, -math.inf):
        o = old.clone()
        o[1] = o[3] = far
        assert all(torch.equal(a, b) for a, b in zip(run(o), want))
    assert want[0].isfinite() and bool(want[2][1].any()) == (kl > 0)
    o[2] = math.nan
    loss, _, g, _ = run(o)
    keep = torch.arange(12, device=dev()) != 2
    assert loss.isnan() and g[2].isnan().all() and torch.equal(g[keep], want[2][keep])
