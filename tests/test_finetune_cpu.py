"""Log-probabilities, the preference and policy losses and clipping without a GPU: the torch
expressions against the definitions in 64 bits, their gradients against differences, what is
refused, which form answers (launches noted, not made)."""
import math

import pytest

torch = pytest.importorskip("torch")
FT = pytest.importorskip("paper_2410_15352_amd.finetune")

bf16, f32, f64 = torch.bfloat16, torch.float32, torch.float64


def _rand(*shape, seed=0, dtype=f64, scale=1.0):
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed + sum(shape)), dtype=f64)).to(dtype)


def _inputs(rows=9, V=7, dtype=f64):
    x = _rand(rows, V, seed=1, dtype=dtype, scale=2.0)
    t = torch.arange(rows) * 3 % V
    t[::4] = -100
    return x, t


def _logp(x, t):
    """By the formula, row by row."""
    out = []
    for row, k in zip(x.double().tolist(), t.tolist()):
        out.append(0.0 if k == -100 else row[k] - math.log(sum(math.exp(v) for v in row)))
    return out


# --------------------------- log-probabilities ------------------------------

def test_logprobs():
    x, t = _inputs()
    assert torch.allclose(FT.token_logprobs(x, t), torch.tensor(_logp(x, t), dtype=f64), atol=1e-13)
    assert torch.autograd.gradcheck(lambda x: FT.token_logprobs(x, t), x.requires_grad_())
    assert FT.token_logprobs(x.detach().to(bf16), t).dtype == f32


def test_logprobs_of_odd_rows():
    x, t = _inputs()
    x[0] = math.nan                        # does not count
    x[1, 0], x[2, int(t[2])] = -math.inf, -math.inf
    x[3] = -math.inf
    t[5], t[6] = 7, -1
    x.requires_grad_()
    l = FT.token_logprobs(x, t)
    assert l[0] == 0 and l[1].isfinite() and l[2] == -math.inf and l[3].isnan() and l[5].isnan() and l[6].isnan()
    (g,) = torch.autograd.grad(l, x, torch.ones_like(l))
    assert torch.equal(g[0], torch.zeros_like(g[0])) and g[1].isfinite().all() and g[5].isnan().all() and g[6].isnan().all()


# --------------------------- preference pairs -------------------------------

def _preference(x, t, starts, ref, beta, eps):
    l = _logp(x, t)
    gain = [0.0 if k == -100 else a - (0.0 if ref is None else float(r))
            for a, k, r in zip(l, t.tolist(), [0.0] * len(l) if ref is None else ref)]
    sums = [sum(gain[a:b]) for a, b in zip(starts, starts[1:])]
    loss = []
    for s0, s1 in zip(sums[::2], sums[1::2]):
        d = beta * (s0 - s1)
        loss.append((1 - eps) * math.log1p(math.exp(-d)) + eps * math.log1p(math.exp(d)))
    return sum(loss) / len(loss), [beta * s for s in sums]


@pytest.mark.parametrize("starts", [[0, 4, 9], [0, 2, 5, 7, 9], [1, 1, 3, 3, 8], [0, 0, 0]], ids=str)
@pytest.mark.parametrize("with_ref", [True, False])
@pytest.mark.parametrize("eps", [0.0, 0.2, 0.5])
def test_preference(starts, with_ref, eps):
    x, t = _inputs()
    ref = _rand(9, seed=3) if with_ref else None
    if with_ref:
        ref[0] = math.nan  # a row that does not count
    loss, rewards = FT.preference_loss(x, t, torch.tensor(starts), reference=ref, beta=0.7, smoothing=eps)
    want, sums = _preference(x, t, starts, ref, 0.7, eps)
    assert math.isclose(float(loss), want, rel_tol=1e-12)
    assert torch.allclose(rewards.reshape(-1), torch.tensor(sums, dtype=f64), atol=1e-12) and not rewards.requires_grad
    assert torch.autograd.gradcheck(
        lambda x: FT.preference_loss(x, t, torch.tensor(starts, dtype=torch.int32), reference=ref, beta=0.7, smoothing=eps)[0],
        x.requires_grad_())


def test_preference_far_apart():
    """Where D is large both the loss and its slope stay numbers."""
    x, t = _inputs()
    for scale in (300.0, -300.0):
        y = (x * 0).requires_grad_()
        ref = torch.where(torch.arange(9) < 5, -scale, scale)
        loss, _ = FT.preference_loss(y, t, torch.tensor([0, 5, 9]), reference=ref, beta=5.0)
        (g,) = torch.autograd.grad(loss, y)
        assert loss.isfinite() and g.isfinite().all()


# -------------------------------- policy ------------------------------------

def _policy_inputs():
    x, t = _inputs(12, 7)
    old = torch.tensor(_logp(x, t), dtype=f64) + _rand(12, seed=5, scale=0.4)
    return x, t, old, _rand(12, seed=6), torch.tensor(_logp(x, t), dtype=f64) + _rand(12, seed=7, scale=0.5)


@pytest.mark.parametrize("kl", [0.0, 0.3])
@pytest.mark.parametrize("clip", [0.2, (0.1, 0.3), (1.0, 0.0)])
def test_policy(kl, clip):
    x, t, old, A, ref = _policy_inputs()
    low, high = clip if isinstance(clip, tuple) else (clip, clip)
    old[0] = A[0] = ref[0] = math.nan  # a row that does not count
    loss, logp = FT.policy_loss(x, t, old, A, reference=ref, clip=clip, kl=kl)
    l, each = _logp(x, t), []
    for i, k in enumerate(t.tolist()):
        if k == -100:
            continue
        r, a = math.exp(l[i] - old[i]), float(A[i])
        d = float(ref[i]) - l[i]
        each.append(-min(r * a, min(max(r, 1 - low), 1 + high) * a) + kl * (math.exp(d) - d - 1))
    assert math.isclose(float(loss), sum(each) / len(each), rel_tol=1e-12)
    assert torch.allclose(logp, torch.tensor(l, dtype=f64), atol=1e-12) and not logp.requires_grad
    assert torch.autograd.gradcheck(lambda x: FT.policy_loss(x, t, old, A, reference=ref, clip=clip, kl=kl)[0], x.requires_grad_())


def test_policy_past_its_bound():
    """A ratio that overflows is clamped away without a trace in the gradient; one that is not, is not."""
    x, t, old, A, _ = _policy_inputs()
    old[1], A[1], old[2], A[2] = -1000.0, 1.0, 1000.0, -1.0
    x.requires_grad_()
    loss, _ = FT.policy_loss(x, t, old, A)
    (g,) = torch.autograd.grad(loss, x)
    assert loss.isfinite() and g.isfinite().all() and not g[1].any() and not g[2].any()


def test_policy_of_no_rows_that_count():
    x, t, old, A, _ = _policy_inputs()
    assert FT.policy_loss(x, torch.full_like(t, -100), old, A)[0].isnan()


def test_constants_pass_no_gradient():
    x, t, old, A, ref = _policy_inputs()
    for v in (x, old, A, ref):
        v.requires_grad_()
    loss, _ = FT.policy_loss(x, t, old, A, reference=ref, kl=0.1)
    assert torch.autograd.grad(loss, (old, A, ref), allow_unused=True) == (None, None, None)
    loss, _ = FT.preference_loss(x, t, torch.tensor([0, 4, 9]), reference=ref)
    assert torch.autograd.grad(loss, ref, allow_unused=True) == (None,)


# ------------------------------- clipping -----------------------------------

def test_clip():
    t = [_rand(3, 4, seed=1), _rand(5, seed=2), _rand(seed=3), torch.zeros(0, dtype=f64)]
    was = [x.clone() for x in t]
    norm = math.sqrt(sum(float((x * x).sum()) for x in was))
    assert math.isclose(float(FT.clip_grad_norm(t)), norm, rel_tol=1e-6) and all(torch.equal(a, b) for a, b in zip(t, was))
    for bound in (norm * 1.01, math.inf):
        FT.clip_grad_norm(t, bound)
        assert all(torch.equal(a, b) for a, b in zip(t, was))
    got = FT.clip_grad_norm([None, *t, t[0]], 0.5)  # one that is given twice counts once
    assert got.dtype == f32 and math.isclose(float(got), norm, rel_tol=1e-6)
    for a, b in zip(t, was):
        assert torch.allclose(a, b * (0.5 / (norm + 1e-6)), rtol=1e-12)
    assert float(FT.clip_grad_norm([], 1.0)) == 0 and float(FT.clip_grad_norm([None])) == 0
    assert float(FT.clip_grad_norm(torch.full((4,), 3.0))) == 6.0
    FT.clip_grad_norm(iter(t), 0.0)
    assert not any(x.any() for x in t)


def test_clip_of_parameters_and_versions():
    p = torch.nn.Parameter(torch.full((4,), 3.0))
    y = p * 1
    z = y.square().sum()
    FT.clip_grad_norm([y], 1.0)
    with pytest.raises(RuntimeError):
        z.backward()  # y was changed
    FT.clip_grad_norm(p, 1.0)
    assert abs(float(p.detach().norm()) - 1) < 1e-5


# ------------------------------- refusals -----------------------------------

_X, _T = torch.zeros(4, 5), torch.zeros(4, dtype=torch.int64)
_S, _R = torch.tensor([0, 2, 4]), torch.zeros(4)


@pytest.mark.parametrize("error,call", [
    (TypeError, lambda: FT.token_logprobs(_X, [0] * 4)),
    (TypeError, lambda: FT.token_logprobs(_X.long(), _T)),
    (TypeError, lambda: FT.token_logprobs(_X, _T.int())),
    (ValueError, lambda: FT.token_logprobs(_X[0], _T)),
    (ValueError, lambda: FT.token_logprobs(_X, _T[:3])),
    (ValueError, lambda: FT.token_logprobs(_X[:0], _T[:0])),
    (ValueError, lambda: FT.token_logprobs(_X[:, :0], _T)),
    (ValueError, lambda: FT.token_logprobs(_X, _T.to("meta"))),
    (TypeError, lambda: FT.preference_loss(_X, _T, [0, 2, 4])),
    (TypeError, lambda: FT.preference_loss(_X, _T, _S, reference=_T)),
    (ValueError, lambda: FT.preference_loss(_X, _T, _S[:2])),
    (ValueError, lambda: FT.preference_loss(_X, _T, torch.tensor([0, 1, 2, 3]))),
    (ValueError, lambda: FT.preference_loss(_X, _T, _S.float())),
    (ValueError, lambda: FT.preference_loss(_X, _T, _S, reference=_R[:3])),
    (ValueError, lambda: FT.preference_loss(_X, _T, _S, beta=0.0)),
    (ValueError, lambda: FT.preference_loss(_X, _T, _S, beta=math.inf)),
    (ValueError, lambda: FT.preference_loss(_X, _T, _S, smoothing=0.6)),
    (ValueError, lambda: FT.preference_loss(_X, _T, _S, smoothing=math.nan)),
    (TypeError, lambda: FT.policy_loss(_X, _T, None, _R)),
    (TypeError, lambda: FT.policy_loss(_X, _T, _R, _T)),
    (ValueError, lambda: FT.policy_loss(_X, _T, _R, _R[:2])),
    (ValueError, lambda: FT.policy_loss(_X, _T, _R, _R.view(4, 1))),
    (ValueError, lambda: FT.policy_loss(_X, _T, _R, _R, kl=0.1)),
    (ValueError, lambda: FT.policy_loss(_X, _T, _R, _R, reference=_R, kl=-0.1)),
    (ValueError, lambda: FT.policy_loss(_X, _T, _R, _R, clip=(1.5, 0.2))),
    (ValueError, lambda: FT.policy_loss(_X, _T, _R, _R, clip=-0.1)),
    (TypeError, lambda: FT.policy_loss(_X, _T, _R, _R, clip=(0.1, 0.2, 0.3))),
    (TypeError, lambda: FT.clip_grad_norm([_T])),
    (TypeError, lambda: FT.clip_grad_norm([3.0])),
    (TypeError, lambda: FT.clip_grad_norm([torch.zeros(3, 3).to_sparse()])),
    (ValueError, lambda: FT.clip_grad_norm([_R], -1.0)),
    (ValueError, lambda: FT.clip_grad_norm([_R], math.nan)),
    (ValueError, lambda: FT.clip_grad_norm([_R, _R.to("meta")], 1.0)),
    (ValueError, lambda: FT.clip_grad_norm([torch.zeros(1).expand(4)], 1.0))])
def test_refuses(error, call):
    with pytest.raises(error):
        call()


def test_rewards_and_logprobs_alone():
    """A backward that no loss reaches."""
    x, t = _inputs()
    loss, rewards = FT.preference_loss(x.requires_grad_(), t, torch.tensor([0, 4, 9]))
    assert loss.requires_grad and not rewards.requires_grad


# -------------------------------- routes ------------------------------------

@pytest.fixture
def launches(monkeypatch):
    names = []
    monkeypatch.setattr(FT, "_here", FT._plain)
    monkeypatch.setattr(FT, "_stream", lambda t: 0)
    monkeypatch.setattr(FT.ops, "_call", lambda name, *args: names.append(name))
    monkeypatch.setattr(FT.ops, "_companion", lambda t, dtype, count: (
        t.dtype == dtype and t.numel() == count and FT._plain(t) and t.is_contiguous()))
    return names


def _fns(x, t):
    starts, rows = torch.tensor([0, 4, 9]), _rand(9, seed=8, dtype=f32)
    return {
        "logprobs": (lambda x: FT._LogprobsFn.apply(x, t).sum(), lambda x: FT.token_logprobs(x, t).sum()),
        "preference": (lambda x: FT._PreferenceFn.apply(x, t, starts, rows, 0.5, 0.1, True)[0],
                       lambda x: FT.preference_loss(x, t, starts, reference=rows, beta=0.5, smoothing=0.1)[0]),
        "policy": (lambda x: FT._PolicyFn.apply(x, t, rows - 2, rows, rows - 2.5, (0.2, 0.3, 0.1))[0],
                   lambda x: FT.policy_loss(x, t, rows - 2, rows, reference=rows - 2.5, clip=(0.2, 0.3), kl=0.1)[0])}


EXPECT = {"logprobs": ["compact_token_logprobs"] * 2,
          "preference": ["compact_token_logprobs", "compact_preference_pairs", "compact_token_logprobs"],
          "policy": ["compact_policy"] * 2}


@pytest.mark.parametrize("which", list(EXPECT))
def test_kernels_answer(launches, which):
    x, t = _inputs(9, 16, bf16)
    x.requires_grad_()
    (g,) = torch.autograd.grad(_fns(x, t)[which][0](x), x)
    assert launches == EXPECT[which] and g.shape == x.shape and g.dtype == bf16


@pytest.mark.parametrize("which", list(EXPECT))
@pytest.mark.parametrize("change", [
    lambda t: t.float() if t.shape == (9, 16) else t,                          # logits of a wider type
    lambda t: t.int() if t.shape == (9,) and t.dtype == torch.int64 else t,    # targets read as int64
    lambda t: torch.stack((t, t), -1)[..., 0] if t.shape == (9,) and t.dtype == torch.int64 else t])
def test_saved_tensors_changed_by_a_hook(launches, which, change):
    x, t = _inputs(9, 16, bf16)
    x.requires_grad_()
    run, plain = _fns(x, t)[which]
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, change):
        y = run(x)
    (g,) = torch.autograd.grad(y, x, torch.tensor(3.0))
    assert launches == EXPECT[which][:-1]
    wide = x.detach().double().requires_grad_()
    (e,) = torch.autograd.grad(plain(wide), wide, torch.tensor(3.0, dtype=f64))
    assert (g.double() - e).abs().max() <= 2.0 ** -7 * e.abs().max()


@pytest.mark.parametrize("which", list(EXPECT))
def test_recorded_backward(launches, which):
    """A backward that is recorded goes by the torch expressions, and may be differentiated again."""
    x, t = _inputs(9, 16, f32)
    x.requires_grad_()
    (g,) = torch.autograd.grad(_fns(x, t)[which][0](x), x, create_graph=True)
    assert launches == EXPECT[which][:-1]
    (h,) = torch.autograd.grad(g.square().sum(), x)
    wide = x.detach().double().requires_grad_()
    (gw,) = torch.autograd.grad(_fns(wide, t)[which][1](wide), wide, create_graph=True)
    (hw,) = torch.autograd.grad(gw.square().sum(), wide)
    assert (h.double() - hw).abs().max() <= 1e-4 * hw.abs().max()


def test_clip_entries(monkeypatch):
    """What the launches are told of each tensor: address, elements, kind; views in any order of dimensions as they are."""
    calls = []
    monkeypatch.setattr(FT, "_devices", lambda t: 0)
    monkeypatch.setattr(FT, "_device_now", lambda: 0)
    monkeypatch.setattr(FT, "_stream", lambda t: 0)
    monkeypatch.setattr(FT, "_clip_pieces", lambda at, n: n)
    monkeypatch.setattr(FT.ops, "_call", lambda name, at, n, *a: calls.append((name, (FT.ctypes.c_uint64 * (3 * n)).from_address(at)[:], a)))
    t = [_rand(4, 6, dtype=bf16), _rand(4, 6, dtype=f32).t(), _rand(3, dtype=f32), _rand(4, 6, dtype=f32)[:, :5]]
    was = t[3].clone()
    FT.clip_grad_norm([*t, None], 1.0)
    name, entries, rest = calls[0]
    assert name == "compact_clip" and rest[:2] == (1.0, True)
    assert entries[:9] == [t[0].data_ptr(), 24, 0, t[1].data_ptr(), 24, 1, t[2].data_ptr(), 3, 1]
    assert entries[9] != t[3].data_ptr() and entries[10:] == [20, 1] and torch.equal(t[3], was)
    FT.clip_grad_norm([t[0], t[2]])
    assert calls[1][1] == [t[0].data_ptr(), 24, 0, t[2].data_ptr(), 3, 1] and calls[1][2][:2] == (0.0, False)
    FT.clip_grad_norm([t[0], t[2].half()], 1.0)
    assert len(calls) == 2


def test_functorch_takes_the_expressions():
    x, t = _inputs()
    g = torch.func.grad(lambda x: FT.policy_loss(x, t, _rand(9, seed=3) - 2, _rand(9, seed=4))[0])(x)
    y = x.clone().requires_grad_()
    (e,) = torch.autograd.grad(FT.policy_loss(y, t, _rand(9, seed=3) - 2, _rand(9, seed=4))[0], y)
    assert torch.allclose(g, e)
    l = torch.func.vmap(lambda x: FT.token_logprobs(x, t))(torch.stack((x, 2 * x)))
    assert torch.allclose(l[1], FT.token_logprobs(2 * x, t))


@pytest.mark.parametrize("forward,backward,held", [(0, 0, True), (7, 7, True), (0, 7, False), (7, 0, False), (7, 8, False)])
def test_the_gradient_held_for_the_backward(launches, monkeypatch, forward, backward, held):
    """The one that the forward formed is given only where both go into the same graph, or into none, and once."""
    where, buffers = [forward], []
    monkeypatch.setattr(FT.ops, "_capture", lambda stream: where[0])
    call = FT._policy_call

    def policy_call(*a, dx=None, unless_one=False, **k):
        buffers.append((dx.data_ptr(), unless_one))
        return call(*a, dx=dx, unless_one=unless_one, **k)

    monkeypatch.setattr(FT, "_policy_call", policy_call)
    x, t = _inputs(9, 16, bf16)
    x.requires_grad_()
    y = _fns(x, t)["policy"][0](x)
    where[0] = backward
    g, h = (torch.autograd.grad(y, x, retain_graph=True)[0] for _ in range(2))
    formed = buffers[0][0]
    assert buffers[1] == (g.data_ptr(), held) and (g.data_ptr() == formed) == held
    assert buffers[2] == (h.data_ptr(), False) and h.data_ptr() != g.data_ptr()


@pytest.mark.parametrize("dtype", [f32, f64])
@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_of_no_advantage(dtype, kl):
    """A row whose advantage is zero has no part but the KL term's, however far its ratio is off; one whose
    ratio is not a number has it all the same."""
    x, t, old, A, ref = _policy_inputs()
    x = x.to(dtype).requires_grad_()
    A[1] = A[2] = 0.0

    def run(old):
        loss, _ = FT.policy_loss(x, t, old, A, reference=ref, kl=kl)
        return loss, torch.autograd.grad(loss, x)[0]

    loss, g = run(old)
    for far in (-1000.0, 1000.0, -math.inf):
        o = old.clone()
        o[1] = far
        assert all(torch.equal(a, b) for a, b in zip(run(o), (loss, g)))
    assert g[1].any() == (kl > 0)
    o[2] = math.nan
    bad, h = run(o)
    assert bad.isnan() and h[2].isnan().all() and h[3].isfinite().all()


@pytest.mark.parametrize("spoil", ["logits", "reference", "target"])
def test_preference_rows_of_no_sequence(spoil):
    """They may hold anything, a target past V too: no part in the loss, and a gradient of zero."""
    x, t = _inputs()
    t[8], starts, ref = 3, torch.tensor([2, 4, 7]), _rand(9, seed=3)

    def run(x, t, ref):
        x = x.clone().requires_grad_()
        loss, rewards = FT.preference_loss(x, t, starts, reference=ref)
        return loss, rewards, torch.autograd.grad(loss, x)[0]

    want = run(x, t, ref)
    x, t, ref = x.clone(), t.clone(), ref.clone()
    for row in (1, 7, 8):
        if spoil == "logits":
            x[row] = math.nan
        elif spoil == "reference":
            ref[row] = math.nan
        else:
            t[row] = 7
    for a, b in zip(run(x, t, ref), want):
        assert torch.equal(a, b)
    assert not want[2][:2].any() and not want[2][7:].any()
