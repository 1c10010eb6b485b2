"""Rows of no sequence in the preference loss: no part in it, whatever they hold, and a gradient of zero."""
import math

import pytest

from gpu_util import dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
FT = pytest.importorskip("paper_2410_15352_amd.finetune")


@pytest.mark.parametrize("route", ["kernels", "expressions"])
@pytest.mark.parametrize("spoil", ["logits", "reference", "target"])
@pytest.mark.parametrize("n", [2, 20])  # in one workgroup, in one of its own for each
def test_rows_of_no_sequence(monkeypatch, route, spoil, n):
    rows, V, dtype = 5 * n + 9, 300, torch.bfloat16 if route == "kernels" else torch.float16
    if route == "kernels":
        monkeypatch.setattr(FT, "_preference_torch", None)
    g = torch.Generator(device=dev()).manual_seed(3)
    x = torch.randn((rows, V), generator=g, device=dev()).to(dtype)
    t = torch.randint(V, (rows,), generator=g, device=dev())
    ref = torch.randn(rows, generator=g, device=dev()) - 6.0
    starts = torch.linspace(4, rows - 5, 2 * n + 1, device=dev()).long()

    def run(x, t, ref):
        x = x.clone().requires_grad_(True)
        loss, rewards = FT.preference_loss(x, t, starts, reference=ref)
        return loss, rewards, torch.autograd.grad(loss, x, torch.full_like(loss, 3.0))[0]

    want = run(x, t, ref)
    for v, bad in ((x, math.nan),) if spoil == "logits" else ((ref, math.nan),) if spoil == "reference" else ((t, V), (t, -3)):
        u = v.clone()
        u[:4], u[-5:] = bad, bad
        for a, b in zip(run(*(u if w is v else w for w in (x, t, ref))), want):
            assert torch.equal(a, b)
    assert want[0].isfinite() and want[2][4:-5].any() and not want[2][:4].any() and not want[2][-5:].any()
