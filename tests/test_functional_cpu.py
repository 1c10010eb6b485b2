"""Rotary positions, windowed attention and distillation without a GPU: the torch
expressions against the definitions written out element by element in 64 bits, their
gradients against differences, and what is refused."""
import math

import pytest

torch = pytest.importorskip("torch")
F = pytest.importorskip("paper_2410_15352_amd.functional")
blk = pytest.importorskip("paper_2410_15352_amd.block")

f64 = torch.float64


def _g(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------- rotary -------------------------------------

@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dims,hd", [(2, 2), (8, 8), (6, 10)])
def test_rotary_by_pairs(layout, dims, hd):
    rope = F.Rotary(dims, base=100.0, layout=layout)
    x = torch.randn(2, 3, 2, hd, generator=_g(1), dtype=f64)
    y, none = rope(x, positions=5), None
    for b in range(2):
        for l in range(3):
            for i in range(dims // 2):
                t = (5 + l) * 100.0 ** (-2 * i / dims)
                p, q = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + dims // 2)
                a, c = x[b, l, :, p], x[b, l, :, q]
                assert torch.allclose(y[b, l, :, p], a * math.cos(t) - c * math.sin(t), atol=1e-12)
                assert torch.allclose(y[b, l, :, q], c * math.cos(t) + a * math.sin(t), atol=1e-12)
    assert torch.equal(y[..., dims:], x[..., dims:])


def test_rotary_scaling():
    f = lambda **k: F.Rotary(64, scaling=k.pop("scaling"), factor=4.0, **k)
    plain = F.Rotary(64).turns(torch.device("cpu"))
    assert torch.allclose(f(scaling="linear").turns(torch.device("cpu")), plain / 4)
    ntk = f(scaling="ntk").turns(torch.device("cpu"))
    assert math.isclose(ntk[0], plain[0]) and math.isclose(ntk[-1], plain[-1] / 4, rel_tol=1e-12)
    parts = f(scaling="parts", original_length=1024, low=1.0, high=32.0)
    t = parts.turns(torch.device("cpu"))
    whole = plain * 1024 >= 32
    none = plain * 1024 <= 1
    assert whole.any() and none.any() and (~whole & ~none).any()
    assert torch.equal(t[whole], plain[whole]) and torch.allclose(t[none], plain[none] / 4)
    between = ~whole & ~none
    assert ((t[between] < plain[between]) & (t[between] > plain[between] / 4)).all()
    assert math.isclose(parts.magnitude, 1 + 0.1 * math.log(4))


def test_rotary_keeps_its_frequencies_under_a_cast():
    rope = F.Rotary(16).to(torch.bfloat16)
    assert rope.turns(torch.device("cpu")).dtype == f64 and not list(rope.parameters()) and not list(rope.buffers())


def test_rotary_gradient():
    rope = F.Rotary(6, layout="half", scaling="parts", factor=2.0, original_length=100)
    q = torch.randn(1, 3, 2, 8, generator=_g(2), dtype=f64, requires_grad=True)
    k = torch.randn(1, 3, 1, 8, generator=_g(3), dtype=f64, requires_grad=True)
    assert torch.autograd.gradcheck(lambda a, b: rope(a, b, positions=torch.tensor([4, 0, 9])), (q, k))


@pytest.mark.parametrize("make", [
    lambda: F.Rotary(3), lambda: F.Rotary(0), lambda: F.Rotary(8, layout="x"), lambda: F.Rotary(8, scaling="x"),
    lambda: F.Rotary(8, factor=0.5), lambda: F.Rotary(2, scaling="ntk", factor=2), lambda: F.Rotary(8, low=3, high=3),
    lambda: F.Rotary(16)(torch.zeros(1, 1, 1, 8)), lambda: F.Rotary(8)(torch.zeros(1, 1, 8)),
    lambda: F.Rotary(8)(torch.zeros(1, 2, 1, 8), torch.zeros(1, 3, 1, 8)),
    lambda: F.Rotary(8)(torch.zeros(1, 2, 1, 8), positions=torch.zeros(3, dtype=torch.int64)),
    lambda: blk.LlamaBlock(64, 4, 64, device="cpu", rope=F.Rotary(32))])
def test_rotary_refuses(make):
    with pytest.raises(ValueError):
        make()


def test_rotary_refuses_types():
    x = torch.zeros(1, 2, 1, 8)
    for args, kw in (((x, x.double()), {}), ((x.long(),), {}), ((x,), dict(positions=torch.zeros(2))), ((x,), dict(positions=1.5))):
        with pytest.raises(TypeError):
            F.Rotary(8)(*args, **kw)


# ------------------------------ attention -----------------------------------

def _by_rows(q, k, v, window, sinks, lengths, scale):
    """The definition, row by row."""
    b, heads, lq, hd = q.shape
    kv, lk = k.shape[1:3]
    o = torch.zeros_like(q)
    for n in range(b):
        L = lk if lengths is None else int(lengths[n])
        for h in range(heads):
            for i in range(lq):
                p = i + L - lq
                js = [j for j in range(L) if j <= p and (window is None or p - j < window or j < sinks)]
                if js:
                    w = torch.softmax(scale * k[n, h * kv // heads, js] @ q[n, h, i], 0)
                    o[n, h, i] = w @ v[n, h * kv // heads, js]
    return o


@pytest.mark.parametrize("heads,kv,lq,lk,window,sinks,lengths", [
    (1, 1, 1, 1, None, 0, None), (4, 2, 5, 5, 2, 1, None), (2, 1, 3, 9, 4, 2, [9, 2]), (3, 3, 7, 4, None, 0, None),
    (2, 2, 6, 6, 1, 0, [0, 6]), (2, 2, 6, 6, 3, 50, [4, 1])])
def test_attention_by_rows(heads, kv, lq, lk, window, sinks, lengths):
    q = torch.randn(2, heads, lq, 8, generator=_g(1), dtype=f64, requires_grad=True)
    k, v = (torch.randn(2, kv, lk, 8, generator=_g(s), dtype=f64, requires_grad=True) for s in (2, 3))
    n = None if lengths is None else torch.tensor(lengths)
    o = F.window_attention(q, k, v, window=window, sinks=sinks, lengths=n, scale=0.7)
    assert torch.allclose(o, _by_rows(q, k, v, window, sinks, lengths, 0.7), atol=1e-12)
    assert torch.autograd.gradcheck(
        lambda *t: F.window_attention(*t, window=window, sinks=sinks, lengths=n, scale=0.7), (q, k, v))


@pytest.mark.parametrize("change", [
    dict(q=(2, 3, 4)), dict(k=(1, 2, 4, 8)), dict(q=(2, 3, 4, 8)), dict(q=(2, 4, 4, 16)), dict(window=0), dict(sinks=-1),
    dict(lengths=torch.tensor([4])), dict(lengths=torch.tensor([4.0, 4.0])), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=math.nan), dict(scale=math.inf)])
def test_attention_refuses(change):
    shapes = dict(q=(2, 4, 4, 8), k=(2, 2, 4, 8), v=(2, 2, 4, 8))
    tensors = {n: torch.zeros(change.get(n, s)) for n, s in shapes.items()}
    with pytest.raises(ValueError):
        F.window_attention(*tensors.values(), **{n: x for n, x in change.items() if n not in shapes})


def test_attention_refuses_types():
    x = torch.zeros(1, 1, 2, 8)
    for t in ((x, x.double(), x), (x.int(), x.int(), x.int())):
        with pytest.raises(TypeError):
            F.window_attention(*t)


def test_attention_splits_rule():
    assert F.attention_splits(16, 16, 16, 1, 4096, 1024, 4) == 4      # 256 waves of rows, 33 tiles
    assert F.attention_splits(4, 32, 8, 1, 70000, F.NO_WINDOW, 0) == 64
    assert F.attention_splits(1, 1, 1, 1, 1, F.NO_WINDOW, 0) == 1
    assert F.attention_splits(4, 16, 16, 4096, 4096, 1024, 4) == 0    # enough rows
    assert F.attention_splits(1 << 16, 1, 1, 1, 4096, 1024, 4) == 0   # past a grid's third dimension
    assert F.attention_splits(1, 16, 4, 1000, 20000, F.NO_WINDOW, 0) == 4  # 128 workgroups of rows
    assert F.attention_splits(1, 16, 4, 1000, 1000, 64, 4) == 0       # too few keys to split


# ----------------------------- distillation ---------------------------------

def _loss_by_rows(x, top, ids, targets, T, w):
    total, n = 0.0, 0
    for r in range(len(x)):
        if targets is not None and targets[r] == -100:
            continue
        n += 1
        e = [k for k in range(ids.shape[1]) if ids[r, k] >= 0 and top[r, k] > -math.inf]
        if e:
            p = torch.softmax(top[r, e] / T, 0)
            q = torch.log_softmax(x[r] / T, 0)
            total = total + w * T * T * sum(p[i] * (torch.log(p[i]) - q[ids[r, k]]) for i, k in enumerate(e))
        if targets is not None:
            total = total - (1 - w) * torch.log_softmax(x[r], 0)[targets[r]]
    return total / n


@pytest.mark.parametrize("T,w", [(1.0, 1.0), (2.0, 0.5), (0.5, 0.0)])
@pytest.mark.parametrize("with_targets", [True, False])
def test_distill_by_rows(T, w, with_targets):
    if w < 1 and not with_targets:
        return
    x = torch.randn(4, 7, generator=_g(1), dtype=f64, requires_grad=True)
    top = torch.randn(4, 3, generator=_g(2), dtype=f64)
    ids = torch.tensor([[1, 2, 3], [6, 0, -1], [-1, -1, -5], [4, 4, 0]])  # missing, none, twice the same
    top[0, 1] = -math.inf
    t = torch.tensor([0, -100, 6, 2]) if with_targets else None
    loss = F.distill_loss(x, top, ids, targets=t, temperature=T, weight=w)
    assert torch.allclose(loss, _loss_by_rows(x, top, ids, t, T, w), atol=1e-12)
    assert torch.autograd.gradcheck(lambda a: F.distill_loss(a, top, ids, targets=t, temperature=T, weight=w), (x,))
    if with_targets:
        (g,) = torch.autograd.grad(loss, x)
        assert torch.equal(g[1], torch.zeros_like(g[1]))


def test_distill_ids_past_the_vocabulary():
    x, top = torch.zeros(2, 5), torch.zeros(2, 1)
    assert F.distill_loss(x, top, torch.tensor([[5], [0]])).isnan()
    assert F.distill_loss(x, top, torch.tensor([[0], [0]]), targets=torch.tensor([5, 0]), weight=0.5).isnan()
    # of a row that does not count, nothing matters
    x[0] = math.nan
    assert F.distill_loss(x, top, torch.tensor([[5], [0]]), targets=torch.tensor([-100, 0]), weight=0.5).isfinite()


@pytest.mark.parametrize("change", [
    dict(logits=torch.zeros(2, 3, 4)), dict(top_logits=torch.zeros(2, 2)), dict(top_logits=torch.zeros(3, 1), top_ids=torch.zeros(3, 1).long()),
    dict(top_logits=torch.zeros(2, 0), top_ids=torch.zeros(2, 0).long()), dict(targets=torch.zeros(3).long()),
    dict(targets=torch.zeros(2)), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.inf),
    dict(temperature=math.nan), dict(weight=1.5), dict(weight=-0.1), dict(weight=math.nan), dict(weight=0.5)])
def test_distill_refuses(change):
    args = dict(logits=torch.zeros(2, 4), top_logits=torch.zeros(2, 1), top_ids=torch.zeros(2, 1).long())
    with pytest.raises(ValueError):
        F.distill_loss(**{**args, **change})


def test_distill_refuses_types():
    x, top, ids = torch.zeros(2, 4), torch.zeros(2, 1), torch.zeros(2, 1).long()
    for t in ((x.int(), top, ids), (x, top.int(), ids), (x, top, top)):
        with pytest.raises(TypeError):
            F.distill_loss(*t)


# -------------------------------- the block ----------------------------------

def test_block_and_model_run_them_together():
    """On the CPU: positions matter, the window cuts, the teacher's loss has a gradient."""
    torch.manual_seed(0)
    rope = F.Rotary(16)
    b = blk.LlamaBlock(64, 2, 64, device="cpu", rope=rope, window=4, sinks=1)
    x = torch.randn(1, 12, 64).to(torch.bfloat16)
    y = b(x)
    far = x.clone()
    far[0, 2] = 0  # token 11 sees 8 .. 11 and 0 (one block: nothing further through it)
    assert torch.equal(b(far)[0, 11], y[0, 11]) and not torch.equal(b(far)[0, 4], y[0, 4])
    first = x.clone()
    first[0, 0] = 0
    assert not torch.equal(b(first)[0, 11], y[0, 11])
    b.rope = None
    assert not torch.equal(b(x), y)
    m = blk.LlamaModel(32, 64, 2, 64, 2, device="cpu", rope=rope, window=4, sinks=1)
    tokens = torch.randint(32, (2, 9))
    loss = m(tokens[:, :-1], tokens[:, 1:], teacher=(torch.randn(2, 8, 3), torch.randint(32, (2, 8, 3))), temperature=2.0)
    loss.backward()
    assert loss.isfinite() and m.head.weight.grad.isfinite().all() and m.embed.grad.abs().sum() > 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.float64])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_attention_leaves_out_what_no_row_sees(dtype, bad):
    """A cache that holds anything past its sequences, and before every row's window."""
    g = torch.Generator().manual_seed(5)
    q = torch.randn(2, 4, 3, 8, generator=g, dtype=dtype).requires_grad_()
    k, v = (torch.randn(2, 2, 20, 8, generator=g, dtype=dtype) for _ in range(2))
    lengths = torch.tensor([11, 3])
    held = [k.clone(), v.clone()]
    for t in held:
        t[0, :, 11:] = bad
        t[1, :, 3:] = bad
        t[0, :, 1:4] = bad  # rows 8, 9, 10 of a window of 5 see 4 on, and the sink 0
    held = [t.requires_grad_() for t in held]
    plain = [t.clone().requires_grad_() for t in (k, v)]
    out = [F.window_attention(q, *kv, window=5, sinks=1, lengths=lengths) for kv in (plain, held)]
    assert torch.equal(out[0], out[1])
    grads = [torch.autograd.grad(o.sum(), (q, *kv)) for o, kv in zip(out, (plain, held))]
    for a, b in zip(*grads):
        assert torch.equal(a, b)
