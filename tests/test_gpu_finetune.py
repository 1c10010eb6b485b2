"""Log-probabilities, the preference and policy losses and clipping on the GPU against float64, at the
edges of chunks, rows, sequences and pieces.

Tolerances.  A term exp(x - m) of a row's sum is off by (1 + |x - m|) 2^-22 of itself, which is at most
2^-21 of the sum's own scale over a row; a sum of V fp32 terms is off by LAM sqrt(V) 2^-24 of itself
besides.  With e the two together a log-probability (put together in fp64) is off by e, and its own
rounding 2^-24 |l|; a softmax's element p by 2 e p; and a gradient g ([v = t] - p) by |dg| + 2 e |g| p,
dg being what g is off by, and by its rounding, at most half a step: 2^-8 of a bf16 result, 2^-24 of
an fp32 one (twice that below, for the sum before it)."""
import math

import pytest

from gpu_util import BF16_U, LAM, U32, dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F = pytest.importorskip("paper_2410_15352_amd.functional")
FT = pytest.importorskip("paper_2410_15352_amd.finetune")
blk = pytest.importorskip("paper_2410_15352_amd.block")

bf16, f32, f64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture
def kernels_only(monkeypatch):
    def no(*a, **k):
        raise AssertionError("torch expressions")
    for name in ("_logprobs_torch", "_preference_torch", "_policy_torch", "_clip_torch"):
        monkeypatch.setattr(FT, name, no)


def _rand(*shape, seed=0, dtype=f32, scale=1.0):
    g = torch.Generator(device=dev()).manual_seed(seed + sum(shape))
    return (scale * torch.randn(shape, generator=g, device=dev())).to(dtype)


def _within(a, ref, tol, what=""):
    bad = ~((a.double() - ref).abs() <= tol + 1e-30)
    assert a.shape == ref.shape and not bool(bad.any()), (what, int(bad.sum()), a.double()[bad][:3], ref[bad][:3])


def _inputs(rows, V, dtype, seed=1):
    """Logits with likely targets at every place of a row, some rows without."""
    x = _rand(rows, V, seed=seed, dtype=dtype, scale=2.0)
    g = torch.Generator(device=dev()).manual_seed(seed)
    t = torch.randint(V, (rows,), generator=g, device=dev())
    t[0], t[-1] = 0, V - 1
    x.scatter_(1, t.unsqueeze(1), (_rand(rows, 1, seed=seed + 1) + math.log(V)).to(dtype))
    if rows > 4:
        t[2::5] = -100
    return x, t


def _reference(x, t):
    """log-probabilities, softmaxes, e of the docstring, which rows count."""
    X = x.detach().double()
    counts = t >= 0
    p = torch.softmax(X, 1)
    l = torch.where(counts, torch.log_softmax(X, 1).gather(1, t.clamp(min=0).unsqueeze(1)).squeeze(1), 0.0)
    return l, p, 2.0 ** -21 + LAM * math.sqrt(x.shape[1]) * U32, counts


def _check_grad(dx, x, t, p, e, g, dg):
    """dx of the gradient g of the rows' log-probabilities, itself off by dg."""
    hot = torch.zeros_like(p).scatter_(1, t.clamp(min=0).unsqueeze(1), 1.0)
    counts = (t >= 0).unsqueeze(1)
    ref = torch.where(counts, g.unsqueeze(1) * (hot - p), 0.0)
    u = BF16_U if x.dtype == bf16 else 2 * U32
    tol = u * ref.abs() + (dg.unsqueeze(1) + 4 * U32 * g.abs().unsqueeze(1)) * (hot + p) + 2 * e * g.abs().unsqueeze(1) * p
    _within(dx, ref, torch.where(counts, tol, 0.0), "dx")


SIZES = [(1, 1), (3, 7), (5, 8), (200, 1003), (33, 2048), (17, 8192), (9, 8201), (6, 32000), (12, 32001), (7, 40000), (5, 70001),
         (3, 131072), (3, 150001)]


# --------------------------- log-probabilities ------------------------------

@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("rows,V", SIZES)
def test_logprobs(kernels_only, rows, V, dtype):
    x, t = _inputs(rows, V, dtype)
    l, p, e, counts = _reference(x, t)
    y = FT.token_logprobs(x, t)
    _within(y, l, e + U32 * l.abs(), "l")
    assert y.dtype == f32 and not y[~counts].any()
    x.requires_grad_(True)
    z = FT.token_logprobs(x, t)
    assert torch.equal(y, z)
    dl = _rand(rows, seed=9)
    if rows > 1:
        dl[-2] = 0.0
    (dx,) = torch.autograd.grad(z, x, dl, retain_graph=True)
    _check_grad(dx, x, t, p, e, dl.double(), torch.zeros_like(l))
    (again,) = torch.autograd.grad(z, x, dl)
    assert torch.equal(dx, again)


@pytest.mark.parametrize("dtype", [bf16, f32])
def test_logprobs_of_odd_rows(kernels_only, dtype):
    """Rows that are not numbers stay alone: they do as the definition does, the others as without them."""
    x, t = _inputs(40, 1003, dtype)
    t[2::5] = 5
    clean = FT.token_logprobs(x, t)
    y = x.clone()
    t[0] = -100
    y[0] = math.nan
    y[1, 7], y[3] = math.nan, -math.inf
    y[4, 9] = math.inf
    y[5, :500] = -math.inf
    y[6, int(t[6])] = -math.inf
    y[7] = 0.0
    t[8], t[9] = 1003, -7
    y.requires_grad_(True)
    l = FT.token_logprobs(y, t)
    assert torch.equal(l[10:], clean[10:]) and l[0] == 0 and l[1].isnan() and l[3].isnan() and l[4].isnan()
    assert l[6] == -math.inf and abs(l[7] + math.log(1003)) < 1e-5 and l[8].isnan() and l[9].isnan()
    (g,) = torch.autograd.grad(l, y, torch.ones_like(l))
    for i in (1, 3, 4, 8, 9):
        assert g[i].isnan().any()
    assert not g[0].any() and g[10:].isfinite().all() and g[5:8].isfinite().all() and not g[5, :500].any()


# --------------------------- preference pairs -------------------------------

def _check_preference(x, t, starts, ref, beta, eps, loss, rewards, dx, factor=1.0):
    l, p, e, counts = _reference(x, t)
    rows, n = x.shape[0], (len(starts) - 1) // 2
    gain = torch.where(counts, l - (0 if ref is None else ref.double()), 0.0)
    off = torch.where(counts, e + U32 * gain.abs(), 0.0)
    spans = [slice(a, b) for a, b in zip(starts, starts[1:])]
    sums, offs = (torch.stack([v[s].sum() for s in spans]).view(n, 2) for v in (gain, off))
    _within(rewards, beta * sums, beta * (offs + U32 * sums.abs()), "rewards")
    D, dD = beta * (sums[:, 0] - sums[:, 1]), beta * offs.sum(1)
    soft = torch.nn.functional.softplus
    each = (1 - eps) * soft(-D) + eps * soft(D)
    _within(loss, each.mean(), (dD + 2 * U32 * each).mean(), "loss")
    slope = factor * beta / n * (torch.sigmoid(D) - (1 - eps))
    ds = abs(factor) * beta / n * dD / 4 + 4 * U32 * slope.abs()
    g, dg = torch.zeros(rows, dtype=f64, device=dev()), torch.zeros(rows, dtype=f64, device=dev())
    for i, s in enumerate(spans):
        g[s], dg[s] = (slope if i % 2 == 0 else -slope)[i // 2], ds[i // 2]
    _check_grad(dx, x, t, p, e, g, dg)


@pytest.mark.parametrize("rows,V,dtype,starts", [
    (2, 7, f32, [0, 1, 2]), (9, 1003, bf16, [0, 4, 9]), (60, 1003, f32, [3, 3, 20, 41, 41, 50, 55]), (700, 500, bf16, [0, 300, 690]),
    (30, 32001, bf16, [0, 7, 15, 20, 30]), (12, 8, f32, [5, 5, 5])], ids=str)
@pytest.mark.parametrize("with_ref,eps,beta", [(True, 0.0, 0.1), (False, 0.1, 0.01), (True, 0.5, 2.0)])
def test_preference(kernels_only, rows, V, dtype, starts, with_ref, eps, beta):
    x, t = _inputs(rows, V, dtype)
    ref = _rand(rows, seed=4, scale=0.5) - 3.0 if with_ref else None
    for kind in (torch.int32, torch.int64):
        x = x.detach().requires_grad_(True)
        loss, rewards = FT.preference_loss(x, t, torch.tensor(starts, device=dev(), dtype=kind), reference=ref, beta=beta, smoothing=eps)
        (dx,) = torch.autograd.grad(loss, x, retain_graph=True)
        _check_preference(x, t, starts, ref, beta, eps, loss.detach(), rewards, dx)
        (dx,) = torch.autograd.grad(loss, x, torch.tensor(-3.0, device=dev()))
        _check_preference(x, t, starts, ref, beta, eps, loss.detach(), rewards, dx, -3.0)
    plain = FT.preference_loss(x.detach(), t, torch.tensor(starts, device=dev()), reference=ref, beta=beta, smoothing=eps)
    assert torch.equal(plain[0], loss) and torch.equal(plain[1], rewards) and not rewards.requires_grad


def test_preference_not_finite(kernels_only):
    """A pair with a row that is not a number, or without a class, spoils the loss and its own gradient alone."""
    x, t = _inputs(40, 100, f32)
    starts = torch.tensor([0, 10, 20, 30, 40], device=dev())
    ref = _rand(40, seed=3)

    def run(x, t, ref):
        x = x.detach().clone().requires_grad_(True)
        loss, rewards = FT.preference_loss(x, t, starts, reference=ref)
        return loss, rewards, torch.autograd.grad(loss, x)[0]

    base = run(x, t, ref)
    for spoil in ("x", "t", "ref"):
        y, u, r = x.detach().clone(), t.clone(), ref.clone()
        u[33] = 5
        want = run(x, u, ref)
        if spoil == "x":
            y[33, 4] = math.nan
        elif spoil == "t":
            u[33] = 100
        else:
            r[33] = math.nan
        loss, rewards, g = run(y, u, r)
        assert loss.isnan() and rewards[1, 1].isnan() and torch.equal(rewards[0], base[1][0])
        assert torch.equal(g[:20], want[2][:20]) and g[33].isnan().any()
    # what does not count may hold anything
    y, r = x.detach().clone(), ref.clone()
    y[t < 0], r[t < 0] = math.nan, math.inf
    for a, b in zip(run(y, t, r), base):
        assert torch.equal(a, b)


def test_preference_starts_out_of_order(kernels_only):
    x, t = _inputs(30, 50, f32)
    x.requires_grad_(True)
    for given, meant in (([-4, 12, 5, 20, 10 ** 6], [0, 12, 12, 20, 30]), ([25, 3, 28], [25, 25, 28])):
        a, b = ([*(o := FT.preference_loss(x, t, torch.tensor(s, device=dev()))), *torch.autograd.grad(o[0], x)] for s in (given, meant))
        for u, v in zip(a, b):
            assert torch.equal(u, v)


def test_preference_far_apart(kernels_only):
    x, t = _inputs(20, 50, f32)
    x.requires_grad_(True)
    for sign in (1, -1):
        ref = torch.where(torch.arange(20, device=dev()) < 10, -500.0 * sign, 500.0 * sign)
        loss, _ = FT.preference_loss(x, t, torch.tensor([0, 10, 20], device=dev()), reference=ref, beta=3.0, smoothing=0.1)
        (g,) = torch.autograd.grad(loss, x)
        assert loss.isfinite() and g.isfinite().all() and g.any()


def test_many_pairs(kernels_only):
    """More starts than a workgroup has threads."""
    x, t = _inputs(1203, 40, f32)
    starts = [0, *range(1, 1200, 2), 1203]
    starts = starts if len(starts) % 2 else starts[:-1] + [1202, 1203]
    ref = _rand(1203, seed=5)
    x.requires_grad_(True)
    loss, rewards = FT.preference_loss(x, t, torch.tensor(starts, device=dev()), reference=ref)
    _check_preference(x, t, starts, ref, 0.1, 0.0, loss.detach(), rewards, torch.autograd.grad(loss, x)[0])


# -------------------------------- policy ------------------------------------

def _policy_inputs(rows, V, dtype, low, high, seed=1):
    x, t = _inputs(rows, V, dtype, seed)
    l, _, _, counts = _reference(x, t)
    ratio = _rand(rows, seed=seed + 2).double() * 0.3
    for border in (1 - low, 1 + high):  # none where rounding decides
        if border > 0:
            ratio = torch.where((torch.exp(ratio) / border - 1).abs() < 1e-3, ratio + 0.01, ratio)
    old = (l - ratio).float()
    return x, t, old, _rand(rows, seed=seed + 3) + 0.3, (l + _rand(rows, seed=seed + 4).double() * 0.5).float()


def _check_policy(x, t, old, A, ref, low, high, kl, loss, logp, dx, factor=1.0):
    l, p, e, counts = _reference(x, t)
    _within(logp, l, e + U32 * l.abs(), "l")
    N, A = counts.sum(), A.double()
    r = torch.exp(l - old.double())
    c = r.clamp(1 - low, 1 + high)
    each = -torch.minimum(r * A, c * A)
    clamped = (A > 0) & (r > 1 + high) | (A < 0) & (r < 1 - low)
    g = torch.where(clamped, 0.0, -A * r)
    # exp is within 2^-22, its argument off by e and its rounding
    er = e + 2.0 ** -21 + U32 * (l - old.double()).abs()
    off = torch.where(clamped, 2 * U32 * each.abs(), er * (A * r).abs())
    dg = torch.where(clamped, 0.0, er * (A * r).abs())
    if kl > 0:
        d = ref.double() - l
        each, g = each + kl * (torch.expm1(d) - d), g - kl * torch.expm1(d)
        ed = kl * ((e + 2.0 ** -21 + U32 * d.abs()) * (torch.exp(d) + 1) + U32 * d.abs())
        off, dg = off + ed, dg + ed
    each, off = torch.where(counts, each, 0.0), torch.where(counts, off, 0.0)
    _within(loss, each.sum() / N, (off + 4 * U32 * each.abs()).sum() / N, "loss")
    _check_grad(dx, x, t, p, e, factor * g / N, abs(factor) * (dg + 8 * U32 * g.abs()) / N)


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("rows,V", SIZES)
@pytest.mark.parametrize("low,high,kl", [(0.2, 0.28, 0.05), (0.2, 0.2, 0.0)])
def test_policy(kernels_only, rows, V, dtype, low, high, kl):
    x, t, old, A, ref = _policy_inputs(rows, V, dtype, low, high)
    x.requires_grad_(True)
    loss, logp = FT.policy_loss(x, t, old, A, reference=ref, clip=(low, high), kl=kl)
    assert not logp.requires_grad
    (dx,) = torch.autograd.grad(loss, x, retain_graph=True)
    _check_policy(x, t, old, A, ref, low, high, kl, loss.detach(), logp, dx)
    (again,) = torch.autograd.grad(loss, x, retain_graph=True)  # the second time formed anew
    assert torch.equal(dx, again)
    (dx,) = torch.autograd.grad(loss, x, torch.tensor(-2.0, device=dev()))
    _check_policy(x, t, old, A, ref, low, high, kl, loss.detach(), logp, dx, -2.0)
    plain = FT.policy_loss(x.detach(), t, old, A, reference=ref, clip=(low, high), kl=kl)
    assert torch.equal(plain[0], loss) and torch.equal(plain[1], logp)


def test_policy_many_rows(kernels_only):
    """More rows than workgroups, with runs of rows that do not count."""
    x, t, old, A, ref = _policy_inputs(5000, 97, bf16, 0.2, 0.2)
    t[1000:2600] = -100
    x.requires_grad_(True)
    loss, logp = FT.policy_loss(x, t, old, A, reference=ref, kl=0.1)
    _check_policy(x, t, old, A, ref, 0.2, 0.2, 0.1, loss.detach(), logp, torch.autograd.grad(loss, x)[0])


def test_policy_not_finite(kernels_only):
    x, t, old, A, ref = _policy_inputs(40, 100, f32, 0.2, 0.2)
    x.requires_grad_(True)

    def run(**with_):
        v = dict(dict(x=x, t=t, old=old, A=A, ref=ref), **with_)
        loss, logp = FT.policy_loss(v["x"], v["t"], v["old"], v["A"], reference=v["ref"], kl=0.1)
        return loss, logp, torch.autograd.grad(loss, v["x"])[0]

    base = run()
    dead = t < 0
    # what does not count may hold anything
    y = x.detach().clone()
    y[dead] = math.nan
    o, a, r = (v.masked_fill(dead, math.nan) for v in (old, A, ref))
    for u, v in zip(run(x=y.requires_grad_(True), old=o, A=a, ref=r), base):
        assert torch.equal(u, v)
    i = int((~dead).nonzero()[3])
    for name, value in (("old", math.nan), ("A", math.nan), ("ref", math.nan), ("t", 100), ("t", -5)):
        v = dict(old=old, A=A, ref=ref, t=t)[name].clone()
        v[i] = value
        loss, logp, g = run(**{name: v})
        assert loss.isnan() and g[i].isnan().all()
        keep = torch.arange(40, device=dev()) != i
        assert torch.equal(g[keep], base[2][keep]) and torch.equal(logp[keep], base[1][keep])
    # a ratio that overflows: clamped away, or not
    v, w = old.clone(), A.clone()
    v[i], w[i] = -1000.0, 1.0
    loss, _, g = run(old=v, A=w)
    assert loss.isfinite() and g.isfinite().all()
    w[i] = -1.0
    assert run(old=v, A=w)[0] == math.inf
    # no row that counts
    loss, logp, g = run(t=torch.full_like(t, -100))
    assert loss.isnan() and not logp.any() and not g.any()


def test_strides_types_and_routes():
    """Logits that are not dense, constants of other types, other types of logits: the same."""
    x, t, old, A, ref = _policy_inputs(30, 300, bf16, 0.2, 0.2)
    starts = torch.tensor([0, 10, 30], device=dev())

    def run(x, t=t, old=old, A=A, ref=ref, starts=starts):
        x = x.detach().requires_grad_(True)
        out = [FT.token_logprobs(x, t), *FT.preference_loss(x, t, starts, reference=ref, beta=0.3),
               *FT.policy_loss(x, t, old, A, reference=ref, kl=0.1)]
        return [*out, *(torch.autograd.grad(y, x, torch.ones_like(y))[0] for y in (out[0], out[1], out[3]))]

    base = run(x)
    wide = torch.zeros(30, 305, dtype=bf16, device=dev())
    wide[:, :300] = x
    off = torch.empty(9003, dtype=bf16, device=dev())[3:].view(30, 300).copy_(x)
    two = lambda v: torch.stack((v, v), 1)[:, 0]
    for got in (run(wide[:, :300]), run(off), run(x.t().contiguous().t()), run(x, two(t), two(old), two(A), two(ref), two(starts)),
                run(x, old=old.double(), A=A.double(), ref=ref.double())):
        for u, v in zip(got, base):
            assert torch.equal(u, v)
    for dtype in (torch.float16, f64):
        for u, v in zip(run(x.to(dtype)), base):
            # (bf16's rounding of the results, and twice the logits' own by fp16)
            assert (u.double() - v.double()).norm() <= 4 * BF16_U * v.double().norm()
    with torch.autocast("cuda", dtype=bf16):
        for u, v in zip(run(x), base):
            assert (u.double() - v.double()).norm() <= 4 * BF16_U * v.double().norm()
    # a recorded backward
    y = x.detach().requires_grad_(True)
    (g,) = torch.autograd.grad(FT.policy_loss(y, t, old, A)[0], y, create_graph=True)
    torch.autograd.grad(g.float().square().sum(), y)


def test_against_differences(kernels_only):
    """The gradients agree with differences of the float64 definition's losses along a direction."""
    x, t, old, A, ref = _policy_inputs(30, 300, f32, 0.2, 0.2)
    starts = [0, 10, 30]
    spans = [slice(a, b) for a, b in zip(starts, starts[1:])]
    counts = t >= 0

    def logp(X):
        return torch.where(counts, torch.log_softmax(X, 1).gather(1, t.clamp(min=0).unsqueeze(1)).squeeze(1), 0.0)

    def preference(X):
        gain = torch.where(counts, logp(X) - ref.double(), 0.0)
        return torch.nn.functional.softplus(-0.3 * (gain[spans[0]].sum() - gain[spans[1]].sum()))

    def policy(X):
        l, a = logp(X), A.double()
        r, d = torch.exp(l - old.double()), ref.double() - l
        each = -torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + 0.1 * (torch.exp(d) - d - 1)
        return each[counts].mean()

    y = x.detach().requires_grad_(True)
    dl = _rand(30, seed=8)
    direction = _rand(30, 300, seed=9).double()
    for loss, plain in (((FT.token_logprobs(y, t) * dl).sum(), lambda X: (logp(X) * dl.double()).sum()),
                        (FT.preference_loss(y, t, torch.tensor(starts, device=dev()), reference=ref, beta=0.3)[0], preference),
                        (FT.policy_loss(y, t, old, A, reference=ref, kl=0.1)[0], policy)):
        (g,) = torch.autograd.grad(loss, y)
        h = 1e-5
        slope = (plain(x.double() + h * direction) - plain(x.double() - h * direction)) / (2 * h)
        # fp32 elements within 2^-18 (V = 300), and the second differences' part h^2
        assert abs((g.double() * direction).sum() - slope) <= 2.0 ** -16 * (g.double() * direction).abs().sum()


def test_other_streams_and_graphs(kernels_only):
    x, t, old, A, ref = _policy_inputs(60, 1003, bf16, 0.2, 0.2)
    x.requires_grad_(True)
    starts, dl = torch.tensor([0, 20, 60], device=dev()), _rand(60, seed=7)
    grads = [_rand(1000, 70, seed=3, dtype=bf16), _rand(33, seed=4)]
    kept = [g.clone() for g in grads]

    def step():
        for g, k in zip(grads, kept):
            g.copy_(k)
        l = FT.token_logprobs(x, t)
        loss, rewards = FT.preference_loss(x, t, starts, reference=ref)
        loss2, logp = FT.policy_loss(x, t, old, A, reference=ref, kl=0.1)
        dx = [torch.autograd.grad(v, x, w)[0] for v, w in ((l, dl), (loss, torch.ones_like(loss)), (loss2 * 2, torch.ones_like(loss)))]
        return [l, loss, rewards, loss2, logp, *dx, FT.clip_grad_norm(grads, 1.0), *grads]

    ref_out = [r.detach().clone() for r in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            out = step()
    torch.cuda.current_stream().wait_stream(s)
    for a, r in zip(out, ref_out):
        assert torch.equal(a, r)
    del out
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        for a in out:
            a.detach().zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, r in zip(out, ref_out):
            assert torch.equal(a, r)
        step()


# ------------------------------- clipping -----------------------------------

def _grads(shapes, seed=1, scale=1.0):
    return [_rand(*shape, seed=seed + i, dtype=dtype, scale=scale) for i, (shape, dtype) in enumerate(shapes)]


def _check_clip(tensors, was, got, bound):
    norm = math.sqrt(sum(float((x.double() ** 2).sum()) for x in was))
    assert abs(float(got) - norm) <= 2 * U32 * norm
    f = 1.0 if bound is None else min(1.0, bound / (norm + 1e-6))
    for x, w in zip(tensors, was):
        if f == 1.0:
            assert torch.equal(x, w)
        else:  # its rounding (half a step of bf16: 2^-7 / 2), the factor's and the fp32 product's
            u = BF16_U if x.dtype == bf16 else 0
            _within(x, w.double() * f, (u + 2 * U32) * w.double().abs() * f + (2.0 ** -134 if u else 2.0 ** -149))


@pytest.mark.parametrize("shapes", [
    [((1,), f32)], [((3,), bf16), ((), f32), ((0, 4), f32)], [((1000, 33), bf16), ((7,), f32), ((129, 255), f32)],
    [((32768,), bf16), ((16384,), f32), ((32769,), bf16)],                       # a piece, and one more
    [((200001,), bf16), ((65537,), f32)],
    [((5,), bf16)] * 400,                                                        # several launches
    [((40, 50), f32 if i % 3 else bf16) for i in range(161)]], ids=lambda s: f"{len(s)}x{s[0][0]}")
def test_clip(kernels_only, shapes):
    tensors = _grads(shapes)
    was = [t.clone() for t in tensors]
    norm = float(sum((x.double() ** 2).sum() for x in was).sqrt())
    for bound in (None, 2 * norm, norm / 3):
        got = FT.clip_grad_norm(tensors, bound)
        _check_clip(tensors, was, got, bound)
        assert torch.equal(got, FT.clip_grad_norm(was))
    FT.clip_grad_norm(tensors, 0.0)
    assert not any(t.any() for t in tensors)


def test_clip_alignments_and_orders(kernels_only):
    """Views from any element on, rows of a wider buffer, other orders of dimensions, one tensor twice; what lies between stays."""
    for first in range(9):
        for count in (1, 6, 7, 8, 9, 1000):
            for dtype in (bf16, f32):
                buf = _rand(1040, seed=first, dtype=dtype)
                was = buf.clone()
                t = buf[first:first + count]
                got = FT.clip_grad_norm([t, None, t], 0.25)
                _check_clip([t], [was[first:first + count]], got, 0.25)
                assert torch.equal(buf[:first], was[:first]) and torch.equal(buf[first + count:], was[first + count:])
    buf = _rand(64, 100, seed=3)
    was = buf.clone()
    t = [buf[:, :30], buf[:, 30:77], _rand(20, 30, seed=4, dtype=bf16).t(), _rand(2, 3, 4, 5, seed=5).permute(2, 0, 3, 1)]
    old = [x.clone() for x in t]
    _check_clip(t, old, FT.clip_grad_norm(t, 1.0), 1.0)
    assert torch.equal(buf[:, 77:], was[:, 77:])


def test_clip_large_and_small_values(kernels_only):
    """Squares outside fp32's range; infinities and NaN."""
    for scale in (1e30, 1e-30):
        t = _grads([((300,), f32), ((300,), bf16)], scale=scale)
        was = [x.clone() for x in t]
        _check_clip(t, was, FT.clip_grad_norm(t, scale), scale)
    t = [torch.full((10,), 3e38, device=dev()), torch.full((10,), 3e38, device=dev())]
    assert FT.clip_grad_norm(t, 1.0).isinf() and (t[0] - 20 ** -0.5).abs().max() < 1e-6  # (the norm passes fp32, the factor does not need it)
    a, b = torch.ones(5, device=dev()), torch.ones(5, device=dev())
    a[2] = math.inf
    assert FT.clip_grad_norm([a, b], 1.0).isinf() and not b.any() and a[2].isnan() and not a[:2].any()
    a, b = torch.ones(5, device=dev()), torch.ones(5, device=dev())
    a[2] = math.nan
    assert FT.clip_grad_norm([a, b], 1.0).isnan() and a.isnan().all() and b.isnan().all()


def test_clip_refuses_and_routes():
    buf = torch.ones(100, device=dev())
    with pytest.raises(ValueError):
        FT.clip_grad_norm([buf[:60], buf[40:]], 1.0)
    with pytest.raises(ValueError):
        FT.clip_grad_norm([torch.ones(1, device=dev()).expand(9)], 1.0)
    assert (buf == 1).all()
    # a mixture with types that the kernels do not take
    t = [torch.full((4,), 3.0, dtype=d, device=dev()) for d in (torch.float16, bf16, f32, f64)]
    assert abs(float(FT.clip_grad_norm(t, 6.0)) - 12) < 1e-5
    for x in t:
        assert (x.double() - 1.5).abs().max() < 1e-5
    y = torch.full((4,), 3.0, device=dev(), requires_grad=True)
    z = y * 1
    loss = z.square().sum()
    FT.clip_grad_norm([z], 1.0)
    with pytest.raises(RuntimeError):
        loss.backward()  # z was changed


# ------------------------- a step of all together ---------------------------

def _model(**k):
    torch.manual_seed(3)
    return blk.LlamaModel(300, 128, 4, 272, 2, rank=16, **k)


@pytest.mark.parametrize("rule", [dict(), dict(rope=True, window=20, sinks=2)], ids=["plain", "rope-window"])
def test_packed_model_is_each_sequence_alone(rule):
    """Packed sequences give each one's logits, and the sum of their gradients."""
    model = _model(**dict(rule, rope=F.Rotary(32) if rule.get("rope") else None))
    lengths = [30, 1, 77]
    starts = torch.tensor([0, 30, 31, 108], device=dev())
    tokens = torch.randint(300, (108,), device=dev())
    packed = model.logits(tokens, starts)
    at = 0
    for n in lengths:
        alone = model.logits(tokens[at:at + n].view(1, n))
        # bf16 layers: each rounding 2^-8 at most; two blocks of seven, the head, on values of the logits' own scale
        assert (packed[at:at + n].double() - alone.double()).norm() <= 16 * BF16_U * alone.double().norm()
        at += n
    loss = model(tokens, tokens.roll(-1), starts=starts)
    loss.backward()
    assert all(p.grad is None or p.grad.isfinite().all() for p in model.parameters())


def _packed_pairs():
    starts = torch.tensor([0, 40, 75, 120, 150], device=dev())
    tokens = torch.randint(300, (150,), device=dev(), generator=torch.Generator(device=dev()).manual_seed(1))
    targets = tokens.roll(-1)
    for s in (0, 40, 75, 120):
        targets[s:s + 10] = -100  # prompts
    targets[starts[1:] - 1] = -100
    return tokens, targets, starts


def test_preference_step(kernels_only, monkeypatch):
    monkeypatch.setattr(F, "_packed_torch", None)
    model = _model(rope=F.Rotary(32))
    tokens, targets, starts = _packed_pairs()
    with torch.no_grad():
        reference = FT.token_logprobs(model.logits(tokens, starts), targets)
    opts = blk.make_optimizers(model, lr=1e-3)
    for step in range(3):
        loss, rewards = FT.preference_loss(model.logits(tokens, starts), targets, starts, reference=reference)
        if step == 0:  # the model is its own reference
            assert abs(float(loss.detach()) - math.log(2)) < 1e-5 and rewards.abs().max() < 1e-4
        loss.backward()
        grads = blk.gradients(model)
        assert len(grads) == len([p for p in model.parameters() if p.numel() > 0]) + 2 * 6
        was = [g.clone() for g in grads]
        _check_clip(grads, was, FT.clip_grad_norm(grads, 0.01), 0.01)
        for o in opts:
            o.step()
            o.zero_grad()
    assert blk.gradients(model) == []


def test_policy_step(kernels_only, monkeypatch):
    monkeypatch.setattr(F, "_packed_torch", None)
    model = _model()
    tokens, targets, starts = _packed_pairs()
    with torch.no_grad():
        old = FT.token_logprobs(model.logits(tokens, starts), targets)
    A = _rand(150, seed=2)
    loss, logp = FT.policy_loss(model.logits(tokens, starts), targets, old, A, reference=old, kl=0.1)
    counts = targets >= 0
    # two sums of the same terms in another order, each within e and its rounding of l (the docstring's), so r
    # is 1 within twice that and the exponential's 2^-21; the loss is -mean A, and the KL term of second order
    off = 2 * (2.0 ** -21 + LAM * math.sqrt(300) * U32 + U32 * float(old.abs().max()))
    assert (logp - old).abs().max() <= off
    assert abs(float(loss.detach()) + float(A[counts].double().mean())) <= (off + 2.0 ** -21) * float(A[counts].abs().mean())
    loss.backward()
    assert FT.clip_grad_norm(blk.gradients(model), 1.0).isfinite()


def test_offsets_past_32_bits(kernels_only):
    """Logits of more than 2^31 elements: the last rows are what they are alone."""
    if torch.cuda.get_device_properties(0).total_memory < 64 << 30:
        pytest.skip("memory")
    rows, V, few = 70001, 32000, 6
    x = torch.zeros(rows, V, dtype=bf16, device=dev())
    x[-few:] = _rand(few, V, seed=1, dtype=bf16, scale=2.0)
    t = torch.full((rows,), -100, device=dev())
    t[-few:] = torch.arange(few, device=dev()) * 1000
    old, A = torch.full((rows,), -11.0, device=dev()), torch.ones(rows, device=dev())
    starts = torch.tensor([0, rows - 3, rows], device=dev())
    x.requires_grad_(True)
    y = x.detach()[-few:].clone().requires_grad_(True)
    last = torch.tensor([0, few - 3, few], device=dev())
    for run in (lambda x, n: FT.token_logprobs(x, t[-n:])[-few:],
                lambda x, n: FT.preference_loss(x, t[-n:], starts if n == rows else last)[0],
                lambda x, n: FT.policy_loss(x, t[-n:], old[-n:], A[-n:], clip=0.9)[0]):
        a, b = run(x, rows), run(y, few)
        (g,), (h,) = torch.autograd.grad(a, x, torch.ones_like(a)), torch.autograd.grad(b, y, torch.ones_like(b))
        assert torch.equal(a, b) and torch.equal(g[-few:], h) and h.any() and not g[:-few].any()
        del a, g


def test_clip_of_a_large_tensor(kernels_only):
    """Elements past 2^31: found and scaled."""
    if torch.cuda.get_device_properties(0).total_memory < 32 << 30:
        pytest.skip("memory")
    t = torch.zeros((1 << 31) + 5, dtype=bf16, device=dev())
    t[-1], t[3] = 3.0, 4.0
    assert float(FT.clip_grad_norm([t], 2.5)) == 5.0
    assert float(t[-1]) == 1.5 and float(t[3]) == 2.0 and float(t.double().sum()) == 3.5


@pytest.mark.parametrize("n,rows", [(16, 300), (17, 300), (2, 16384), (2, 16385)])
def test_pairs_on_both_sides_of_the_rule(kernels_only, n, rows):
    x, t = _inputs(rows, 24, f32)
    starts = [i * rows // (2 * n) for i in range(2 * n + 1)]
    ref = _rand(rows, seed=4, scale=0.2) - 3.0
    x.requires_grad_(True)
    loss, rewards = FT.preference_loss(x, t, torch.tensor(starts, device=dev()), reference=ref, beta=0.05, smoothing=0.2)
    _check_preference(x, t, starts, ref, 0.05, 0.2, loss.detach(), rewards, torch.autograd.grad(loss, x)[0])


@pytest.mark.parametrize("n", [FT.OWN_PAIRS, FT.OWN_PAIRS + 1, 4500])
def test_pairs_on_both_sides_of_the_bounds_launch(kernels_only, n):
    """Starts' running maximum by each pair, and before all of them: 4500 pairs take more than one
    round of 4096 starts."""
    rows = 3 * n
    x, t = _inputs(rows, 8, f32)
    starts = [2 + i * (rows - 5) // (2 * n) for i in range(2 * n + 1)]
    ref = _rand(rows, seed=4, scale=0.2) - 2.0
    x.requires_grad_(True)
    loss, rewards = FT.preference_loss(x, t, torch.tensor(starts, device=dev()), reference=ref, beta=0.05, smoothing=0.2)
    (dx,) = torch.autograd.grad(loss, x)
    _check_preference(x, t, starts, ref, 0.05, 0.2, loss.detach(), rewards, dx)
    # out of order, of 32 bits, not dense
    given = torch.tensor(starts, device=dev(), dtype=torch.int32)
    meant = given.clone()
    given[1000], given[4095], given[-3] = rows + 9, -7, 0
    apart = torch.stack([given, given + 1], 1)[:, 0]
    out = FT.preference_loss(x, t, apart, reference=ref)
    meant[1000:] = rows
    for a, b in zip((*out, *torch.autograd.grad(out[0], x)), (*(o := FT.preference_loss(x, t, meant, reference=ref)), *torch.autograd.grad(o[0], x))):
        assert torch.equal(a, b)


def test_a_million_pairs(kernels_only):
    """Most of them empty: their reward is 0, their loss log 2."""
    n, rows = 1 << 20, 64
    x, t = _inputs(rows, 50, f32)
    l, _, e, _ = _reference(x, t)
    at = torch.arange(rows, device=dev()) * 1009
    starts = torch.searchsorted(at, torch.arange(2 * n + 1, device=dev()))
    loss, rewards = FT.preference_loss(x, t, starts, beta=1.0)
    sums = torch.zeros(2 * n, dtype=f64, device=dev())
    sums[at] = l  # row i is the sequence between two starts that differ by it
    _within(rewards, sums.view(n, 2), (e + 2 * U32 * l.abs().max()) * (sums != 0).view(n, 2), "rewards")
    D = sums[0::2] - sums[1::2]
    _within(loss, torch.nn.functional.softplus(-D).mean(), 2 * e * (rows / n) + 2 * U32, "loss")
