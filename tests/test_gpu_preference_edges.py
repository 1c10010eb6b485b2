"""Edges of the preference loss on the GPU: rows of no sequence, which have no part whatever they hold and a
gradient of zero, and pairs on both sides of a rule."""
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


@pytest.mark.parametrize("n,rows", [(1, 4096), (1, 4097), (2, 8192), (2, 8193), (4, 16384), (16, 16384)])
def test_pairs_on_both_sides_of_the_rows_each(monkeypatch, n, rows):
    """A wave to a pair up to 4096 rows of each, a workgroup past that.  Sums of exact numbers: l = -log V in
    every row, equal in fp64 whatever their order, and a reference of multiples of 2^-6."""
    monkeypatch.setattr(FT, "_preference_torch", None)
    V = 8
    x = torch.zeros(rows, V, device=dev()).requires_grad_(True)
    g = torch.Generator(device=dev()).manual_seed(3)
    t = torch.randint(V, (rows,), generator=g, device=dev())
    ref = torch.randint(-400, 0, (rows,), generator=g, device=dev()) / 64.0
    ends = [i * rows // (2 * n) for i in range(2 * n + 1)]
    loss, rewards = FT.preference_loss(x, t, torch.tensor(ends, device=dev()), reference=ref, beta=2.0 ** -9)
    l = FT.token_logprobs(x.detach(), t)
    gain = l.double() - ref.double()
    sums = torch.stack([gain[a:b].sum() for a, b in zip(ends, ends[1:])]).view(n, 2) * 2.0 ** -9
    # rows of fp32: gain is rounded once, by at most half a step
    off = 2.0 ** -9 * rows / (2 * n) * 2.0 ** -24 * float(gain.abs().max()) + 2.0 ** -24 * sums.abs()
    assert ((rewards.double() - sums).abs() <= off).all()
    D = sums[:, 0] - sums[:, 1]
    want = torch.nn.functional.softplus(-D).mean()
    assert (loss.detach().double() - want).abs() <= 2 * off.max() + 2.0 ** -23 * want
    (dx,) = torch.autograd.grad(loss, x)
    slope = 2.0 ** -9 / n * (torch.sigmoid(D) - 1)
    each = torch.cat([torch.full((b - a,), float(slope[i // 2]) * (1 if i % 2 == 0 else -1), dtype=torch.float64, device=dev())
                      for i, (a, b) in enumerate(zip(ends, ends[1:]))])
    hot = torch.zeros(rows, V, dtype=torch.float64, device=dev()).scatter_(1, t.unsqueeze(1), 1.0)
    # the slope's error: beta / n times what D is off by, over 4; its and the softmax's fp32 steps
    tol = 2.0 ** -9 / n * 2 * float(off.max()) / 4 + 2.0 ** -20 * each.abs().unsqueeze(1)
    assert ((dx.double() - each.unsqueeze(1) * (hot - 1 / V)).abs() <= tol).all()
