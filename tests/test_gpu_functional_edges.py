"""Rotary positions, windowed attention and distillation on the GPU where a call is unusual:
first under a capture, of very many or very few rows, with keys of infinities."""
import math

import pytest

from gpu_util import dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F = pytest.importorskip("paper_2410_15352_amd.functional")
whole = pytest.importorskip("test_gpu_functional")


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


def _corners(got, q, k, v, do, window, sinks, lengths=None):
    """The first and the last heads of k against float64, under the bounds of test_gpu_functional."""
    G = q.shape[1] // k.shape[1]
    for b, h in ((slice(0, 1), 0), (slice(-1, None), k.shape[1] - 1)):
        qs, ks = slice(h * G, (h + 1) * G), slice(h, h + 1)
        part = [t[b, s].detach() for t, s in zip(got, (qs, qs, ks, ks))]
        whole._check(part, q[b, qs], k[b, ks], v[b, ks], do[b, qs], window, sinks, None if lengths is None else lengths[b],
                     q.shape[3] ** -0.5, names=" ".join("o dq dk dv".split()[:len(got)]))


@pytest.mark.parametrize("b,heads,kv,l,hd,window,sinks", [
    (16, 16, 16, 700, 64, 31, 300),   # sinks' blocks enough: one workgroup walks all rows past their windows
    (2, 8, 4, 1300, 128, 40, 257),
    (3, 4, 4, 900, 32, 100, 799)])    # one key short of all
def test_attention_gradients_of_many_sinks(b, heads, kv, l, hd, window, sinks):
    q = _rand(b, heads, l, hd, seed=1).requires_grad_(True)
    k, v = (_rand(b, kv, l, hd, seed=s).requires_grad_(True) for s in (2, 3))
    do = _rand(b, heads, l, hd, seed=4)
    o = F.window_attention(q, k, v, window=window, sinks=sinks)
    _corners((o, *torch.autograd.grad(o, (q, k, v), do)), q, k, v, do, window, sinks)


def test_attention_of_sinks_that_reach_the_window():
    q, k, v, do = (_rand(2, 2, 300, 64, seed=s) for s in range(4))

    def run(**rule):
        t = [x.clone().requires_grad_(True) for x in (q, k, v)]
        o = F.window_attention(*t, **rule)
        return [o, *torch.autograd.grad(o, t, do)]

    for a, c in zip(run(window=100, sinks=200), run()):
        assert torch.equal(a, c)


def test_attention_of_very_many_short_sequences():
    """2^24 rows of 32 to a head: more than are joined, no ranges of keys then."""
    b, heads, kv, l, hd = 4096, 128, 8, 32, 8
    q = _rand(b, heads, l, hd, seed=1).requires_grad_(True)
    k, v = (_rand(b, kv, l, hd, seed=s).requires_grad_(True) for s in (2, 3))
    do = _rand(b, heads, l, hd, seed=4)
    o = F.window_attention(q, k, v, window=9, sinks=1)
    _corners((o, *torch.autograd.grad(o, (q, k, v), do)), q, k, v, do, 9, 1)


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_rows_whose_scores_are_all_minus_infinity(monkeypatch, hd):
    """What a row sees propagates: the softmax of nothing but -inf is NaN.  A row that sees no key is zero."""
    b, h, l, window = 2, 2, 200, 4
    q, do = _rand(b, h, l, hd, seed=1).abs() + 0.5, _rand(b, h, l, hd, seed=2)
    k, v = _rand(b, h, l, hd, seed=3), _rand(b, h, l, hd, seed=4)
    k[:, :, 50:61] = -math.inf
    k[:, :, 190:] = -math.inf
    lengths = torch.tensor([l, 40], device=dev())  # the second's first 160 rows see nothing
    for lq, splits, few in ((l, 0, 0), (l, 3, 0), (l, 70, 0), (3, 1, 128), (3, 2, 128)):
        monkeypatch.setattr(F, "attention_splits", lambda *a: splits)
        monkeypatch.setattr(F, "FEW_ROWS", few)
        qs = q[:, :, -lq:]
        o = F.window_attention(qs, k, v, window=window, lengths=lengths)
        expect = F._attention_torch(qs.double(), k.double(), v.double(), window, 0, lengths, hd ** -0.5)
        assert torch.equal(o.isnan(), expect.isnan())
        assert bool(o[0, :, -3:].isnan().all()) and (lq < l or bool((o[1, :, :160] == 0).all()))
        if lq == l:
            assert o[0, 0, :, 0].isnan().sum() == 8 + 7 and not o[1].isnan().any()
    monkeypatch.undo()
    t = [x.clone().requires_grad_(True) for x in (q, k, v)]
    dq, dk, dv = torch.autograd.grad(F.window_attention(*t, window=window), t, do)
    rows = torch.zeros(l, dtype=torch.bool, device=dev())
    rows[53:61], rows[193:] = True, True               # rows of such keys alone
    touched = torch.zeros_like(rows)
    touched[50:64], touched[190:] = True, True         # and those that see one of them
    assert bool(dq[:, :, rows].isnan().all()) and not dq[:, :, ~touched].isnan().any()
    keys = torch.zeros_like(rows)
    keys[50:61], keys[190:] = True, True
    assert bool(dk[:, :, keys].isnan().all()) and bool(dv[:, :, keys].isnan().all())
    far = ~touched
    far[47:50], far[187:190] = False, False            # (seen by rows that see such a key)
    assert not dk[:, :, far].isnan().any() and not dv[:, :, far].isnan().any()


@pytest.mark.parametrize("rank", [None, 16])
def test_projection_seen_by_a_hook_is_not_rotated(rank):
    blk = pytest.importorskip("paper_2410_15352_amd.block")
    torch.manual_seed(0)
    b = blk.LlamaBlock(128, 2, 256, rank=rank, rope=F.Rotary(64), window=20)
    x, dy = _rand(2, 100, 128).requires_grad_(True), _rand(2, 100, 128, seed=1)
    plain = [b(x), *torch.autograd.grad(b(x), x, dy)]
    kept = []
    b.qkv.register_forward_hook(lambda m, i, o: kept.append((o, o.detach().clone())))
    seen = [b(x), *torch.autograd.grad(b(x), x, dy)]
    assert all(torch.equal(a, c) for a, c in kept)
    for a, c in zip(seen, plain):
        assert torch.equal(a, c)


@pytest.mark.parametrize("l,rope", [(256, True), (256, False), (33, True)])
def test_block_saved_activations_with_a_window(l, rope):
    """What the list says a block with windowed attention keeps is what autograd keeps."""
    nn = pytest.importorskip("test_gpu_nn")
    blk = nn.blk_mod
    b, d, heads, ffn = 3, 192, 3, 256
    for rank in (None, 24):
        block = blk.LlamaBlock(d, heads, ffn, rank=rank, rope=F.Rotary(64) if rope else None, window=20, sinks=1)
        x = _rand(b, l, d).requires_grad_(True)
        block(x).float().sum().backward()
        assert nn._saved_bytes(block, x)[0] == blk.block_saved_bytes(b, l, d, heads, ffn, rank=rank, window=20)


def test_attention_over_no_keys():
    q = _rand(2, 4, 3, 64).requires_grad_(True)
    k, v = (torch.empty(2, 2, 0, 64, dtype=q.dtype, device=dev(), requires_grad=True) for _ in range(2))
    o = F.window_attention(q, k, v)
    grads = torch.autograd.grad(o, (q, k, v), torch.ones_like(o))
    assert not o.any() and not grads[0].any() and grads[1].shape == k.shape and grads[2].shape == v.shape


@pytest.mark.parametrize("lq,lk,splits,few", [(300, 300, None, None), (32, 200, None, None), (300, 300, 3, 0)],
                         ids=["rows", "waves, joined", "workgroups, joined"])
@pytest.mark.parametrize("hd", [64, 80, 128])
def test_attention_gradients_of_few_keys_keep_their_digits(monkeypatch, hd, lq, lk, splits, few):
    """Of rows of 4 keys dq and dk are nearly as good as the exact ones rounded to bf16: dS goes in
    two parts and D knows o to 16 bits.

    In 64 bits with these roundings put in (P to bf16 among them) the error is 1.09 to 1.12 times that
    of the rounded exact gradients.  dS in one part makes it 1.47 to 1.54, o rounded to bf16 alone
    1.35 to 1.54; the bound lies between."""
    if splits is not None:
        monkeypatch.setattr(F, "attention_splits", lambda *a: splits)
        monkeypatch.setattr(F, "FEW_ROWS", few)
    q, do = (_rand(4, 8, lq, hd, seed=s) for s in (1, 2))
    k, v = (_rand(4, 4, lk, hd, seed=s) for s in (3, 4))
    t = [x.clone().requires_grad_(True) for x in (q, k, v)]
    got = torch.autograd.grad(F.window_attention(*t, window=4), t, do)
    ref = whole._reference(q, k, v, do, 4, 0, None, hd ** -0.5)[0][1:]
    for name, g, r in zip(("dq", "dk"), got, ref):
        least = (r.to(torch.bfloat16).double() - r).norm()
        assert (g.cpu().double() - r).norm() <= 1.2 * least, (name, float((g.cpu().double() - r).norm() / least))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_attention_values_that_are_seen_propagate_however_small_their_weight(monkeypatch, hd, value):
    """A key whose score lies 400 below the row's largest has a weight that fp32 does not hold;
    its infinity or NaN is in the row's mean all the same, before the large score as after it."""
    l = 200
    q = torch.zeros(1, 2, l, hd, dtype=torch.bfloat16, device=dev())
    q[..., 0] = 20
    k, v = torch.zeros_like(q), _rand(1, 2, l, hd, seed=1)
    k[..., 150, 0] = 20                      # a score of 400 from row 150 on
    v[:, 0, 3, 5], v[:, 1, 170, 5] = value, value
    rows = torch.arange(l, device=dev())
    for lq, splits, few in ((l, 0, 0), (l, 2, 0), (l, 3, 0), (3, 1, 128), (3, 3, 128)):
        monkeypatch.setattr(F, "attention_splits", lambda *a: splits)
        monkeypatch.setattr(F, "FEW_ROWS", few)
        o = F.window_attention(q[:, :, -lq:], k, v, window=198, sinks=2, scale=1.0)
        hit = torch.zeros(2, l, dtype=torch.bool, device=dev())
        hit[0], hit[1] = rows >= 3, rows >= 170
        hit = hit[:, -lq:]
        assert torch.equal(~o[0, ..., 5].isfinite(), hit), (lq, splits)
        others = torch.arange(hd, device=dev()) != 5
        assert bool(o[..., others].isfinite().all())


def test_saved_tensors_kept_on_the_host():
    """save_on_cpu gives back dense copies: the same gradients."""
    rope = F.Rotary(64)
    q, k, v, do = (_rand(2, 70, n, 64, seed=s) for s, n in enumerate((4, 2, 2, 4)))
    lengths, pos = torch.tensor([70, 31], device=dev()), torch.arange(70, device=dev())
    x, top = _rand(9, 1001), _rand(9, 5, seed=1)
    ids, targets = torch.arange(45, device=dev()).view(9, 5) * 20, torch.arange(9, device=dev())

    def run():
        t = [y.clone().requires_grad_(True) for y in (q, k, v)]
        z = x.clone().requires_grad_(True)
        rq, rk = rope(t[0], t[1], positions=pos)
        o = F.window_attention(rq.transpose(1, 2), rk.transpose(1, 2), t[2].transpose(1, 2), window=20, sinks=1, lengths=lengths)
        loss = F.distill_loss(z, top, ids, targets=targets, temperature=2.0, weight=0.5)
        return lambda: torch.autograd.grad((o, loss), (*t, z), (do.transpose(1, 2), torch.tensor(3.0, device=dev())))

    plain = run()()
    with torch.autograd.graph.save_on_cpu():
        back = run()
    for a, c in zip(back(), plain):
        assert torch.equal(a, c)
