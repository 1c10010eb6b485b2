"""Log-probabilities of tokens that are nearly certain: a term of 1 and V - 1 terms of exp(-17.5), each less than
half a unit in the last place of an fp32 sum past 1, that must not be lost one by one.

Tolerance.  A term is off by 2^-22 of itself (the exponential) and 17.5 times 2^-24 twice and 2^-26 (its argument: a
difference, a product, the constant): 2.6e-6, of terms that make up w of the sum.  A sum of fp32 terms takes at most
7 + 3 additions before it is added in fp64, each off by half a unit in the last place at most: 10 x 2^-24 of a sum of at
least 1.  The result's own rounding is 2^-24 |l|."""
import math

import pytest

from gpu_util import dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
FT = pytest.importorskip("paper_2410_15352_amd.finetune")

LEAST = -17.5


def _row(V, dtype, places):
    x = torch.full((len(places), V), LEAST, device=dev(), dtype=dtype)
    t = torch.tensor(places, device=dev())
    x[torch.arange(len(places), device=dev()), t] = 0.0
    rest = (V - 1) * math.exp(LEAST)
    l = -math.log1p(rest)
    return x, t, l, 10 * 2.0 ** -24 + 2.6e-6 * rest / (1 + rest) - 2.0 ** -24 * l


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [7, 1003, 8200, 32000, 65536, 131072, 150001, 1 << 20])
def test_nearly_certain_tokens(monkeypatch, V, dtype):
    for name in ("_logprobs_torch", "_policy_torch", "_preference_torch"):
        monkeypatch.setattr(FT, name, None)
    places = [0, V - 1, V // 2, V // 3, min(V - 1, 1001)]
    x, t, l, tol = _row(V, dtype, places)
    rows = len(places)
    ones = torch.ones(rows, device=dev())
    y = FT.token_logprobs(x, t)
    assert (y.double() - l).abs().max() <= tol
    _, z = FT.policy_loss(x, t, 0 * ones, ones)
    assert (z.double() - l).abs().max() <= tol
    reference = torch.full((rows,), l, device=dev())
    left = l - float(reference[0].double())  # of l in fp32
    starts = torch.tensor([0, 2, rows], device=dev())
    _, rewards = FT.preference_loss(x, t, starts, reference=reference, beta=1.0)
    want = torch.tensor([2 * left, (rows - 2) * left], device=dev(), dtype=torch.float64)
    assert ((rewards[0].double() - want).abs() <= (1 + 2.0 ** -23) * torch.tensor([2, rows - 2], device=dev()) * tol).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_of_nearly_certain_tokens(monkeypatch, dtype):
    """The target's element is g (1 - p): a difference of near numbers, from the same sum."""
    monkeypatch.setattr(FT, "_logprobs_torch", None)
    V = 131072
    x, t, l, tol = _row(V, dtype, [0, V - 1, 70000])
    x.requires_grad_(True)
    (dx,) = torch.autograd.grad(FT.token_logprobs(x, t).sum(), x)
    # p off by tol and the roundings of the sum, the factor, the exponential and the product; dx's own
    at = dx.gather(1, t.unsqueeze(1)).double()
    assert (at + math.expm1(l)).abs().max() <= tol + 5 * 2.0 ** -24 + torch.finfo(dtype).eps / 2 * -math.expm1(l)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [3000, 32000])
def test_long_sums_do_not_drift(monkeypatch, dtype, V):
    """The roundings of a row's terms are to the nearest, of either sign: over thousands of rows a sum of differences to
    the exact log-probabilities grows by less than a quarter of fp32's half step past 1, 2^-26, a row.  (The hardware's
    exponential is off by 3.4e-9 on the mean, and a row's l by 4e-8 around its own, 4e-8 / sqrt(2000) on the mean: together
    4.3e-9, and three times the second part still under 7e-9.)"""
    monkeypatch.setattr(FT, "_preference_torch", None)
    rows = 4000
    g = torch.Generator(device=dev()).manual_seed(V)
    x = (2.0 * torch.randn(rows, V, generator=g, device=dev())).to(dtype)
    t = torch.randint(V, (rows,), generator=g, device=dev())
    x.scatter_(1, t.unsqueeze(1), (2.0 * torch.randn(rows, 1, generator=g, device=dev()) + math.log(V) + 1.0).to(dtype))
    l = torch.cat([torch.log_softmax(a.double(), 1).gather(1, b.unsqueeze(1)).squeeze(1) for a, b in zip(x.split(500), t.split(500))])
    reference = l.float()
    left = (l - reference.double()).view(2, -1).sum(1)
    _, rewards = FT.preference_loss(x, t, torch.tensor([0, rows // 2, rows], device=dev()), reference=reference, beta=1.0)
    assert ((rewards[0].double() - left).abs() <= rows // 2 * 2.0 ** -26).all()
