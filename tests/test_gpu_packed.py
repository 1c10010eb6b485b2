"""Attention over packed sequences on the GPU, sequence by sequence against float64 with the bounds
that test_gpu_functional.py derives for attention, at the edges of tiles, sequences and spans."""
import math

import pytest

from gpu_util import dev
from test_gpu_functional import _rand, _reference, _within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F = pytest.importorskip("paper_2410_15352_amd.functional")


@pytest.fixture
def kernels_only(monkeypatch):
    def no(*a, **k):
        raise AssertionError("torch expressions")
    monkeypatch.setattr(F, "_packed_torch", no)


def _inputs(rows, heads, kv, hd, seed=1):
    q = _rand(rows, heads, hd, seed=seed).requires_grad_(True)
    k, v = (_rand(rows, kv, hd, seed=seed + s).requires_grad_(True) for s in (1, 2))
    return q, k, v, _rand(rows, heads, hd, seed=seed + 3)


def _check(got, q, k, v, do, starts, window, sinks, scale=None):
    hd = q.shape[2]
    scale = hd ** -0.5 if scale is None else scale
    inside = torch.zeros(q.shape[0], dtype=torch.bool)
    for a, b in zip(starts, starts[1:]):
        if a == b:
            continue
        inside[a:b] = True
        padded = [t.detach()[a:b].transpose(0, 1).unsqueeze(0) for t in (q, k, v, do)]
        refs, tols = _reference(*padded, window, sinks, None, scale)
        for name, x, r, t in zip(("o", "dq", "dk", "dv"), got, refs, tols):
            _within(x.detach()[a:b].transpose(0, 1).unsqueeze(0).cpu(), r, t, (name, a, b))
    for x in got:
        assert not x.detach().cpu()[~inside].any()


CASES = [
    # heads, kv, hd, rows, starts, window, sinks
    (1, 1, 8, 1, [0, 1], None, 0),
    (2, 1, 24, 40, [0, 1, 2, 35, 40], None, 0),                  # single rows, shared keys
    (4, 2, 64, 300, [5, 70, 70, 199, 299], 7, 3),                # gaps before and behind, an empty sequence
    (2, 2, 128, 700, [0, 128, 256, 513, 700], 64, 70),           # ends on a tile's, more sinks than the window
    (2, 1, 96, 513, [0, 513], 1, 0),                             # each row sees itself
    (6, 2, 64, 900, [0, 129, 130, 870], 129, 1),
    (5, 1, 80, 800, [0, 700, 765, 800], 301, 1),                 # heads that share keys by fives
    (8, 8, 64, 1400, [0, 1100, 1400], 600, 70),                  # rows that see more than 512 keys, sinks of two blocks
    (1, 1, 128, 1100, [100, 1100], 200, 130),
    (16, 4, 104, 1500, [0, 1400, 1490], None, 0),
    (3, 3, 32, 200, list(range(0, 201, 2)), None, 0),            # a hundred sequences of two rows
    (2, 1, 64, 260, [0, 260], 20, 200),                          # sinks' rows as many as the rows
    (2, 2, 128, 500, [0, 200, 400, 450], 30, 160),
    (2, 1, 64, 50, [0, 0, 0], None, 0),                          # no sequence has a row
    (2, 1, 64, 50, [50, 50], 3, 1),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_packed(kernels_only, case):
    heads, kv, hd, rows, starts, window, sinks = case
    q, k, v, do = _inputs(rows, heads, kv, hd)
    for dtype in (torch.int32, torch.int64):
        o = F.packed_attention(q, k, v, torch.tensor(starts, dtype=dtype, device=dev()), window=window, sinks=sinks)
        grads = torch.autograd.grad(o, (q, k, v), do)
        _check((o, *grads), q, k, v, do, starts, window, sinks)
        again = F.packed_attention(q, k, v, torch.tensor(starts, dtype=dtype, device=dev()), window=window, sinks=sinks)
        assert torch.equal(o, again)  # and so the gradients
        for x, y in zip(grads, torch.autograd.grad(again, (q, k, v), do)):
            assert torch.equal(x, y)
        plain = F.packed_attention(q.detach(), k.detach(), v.detach(), torch.tensor(starts, dtype=dtype, device=dev()),
                                   window=window, sinks=sinks)
        assert torch.equal(o, plain)


def test_as_window_attention_of_each(kernels_only):
    """A sequence among others is what it is alone, bit for bit (forward; the sums of gradients may be split otherwise)."""
    starts = [0, 333, 340, 1000]
    q, k, v, _ = _inputs(1024, 4, 2, 64)
    o = F.packed_attention(q, k, v, torch.tensor(starts, device=dev()), window=100, sinks=3)
    for a, b in zip(starts, starts[1:]):
        one = F.packed_attention(q[a:b], k[a:b], v[a:b], torch.tensor([0, b - a], device=dev()), window=100, sinks=3)
        assert torch.equal(o[a:b], one)


def test_sequences_do_not_meet(kernels_only):
    """A NaN in one sequence, or in rows of none, leaves the others as they are, and their gradients."""
    starts = torch.tensor([3, 150, 200, 390], device=dev())
    q, k, v, do = _inputs(400, 2, 2, 64)

    def run(*t):
        t = [x.detach().clone().requires_grad_(True) for x in t]
        o = F.packed_attention(*t, starts, window=90, sinks=2)
        return o, *torch.autograd.grad(o, t, do)

    base = run(q, k, v)
    keep = torch.ones(400, dtype=torch.bool, device=dev())
    keep[150:200] = False
    for value in (math.nan, math.inf, -math.inf):
        bad = [t.detach().clone() for t in (q, k, v)]
        for t in bad:
            t[160:170] = value
            t[:3], t[390:] = value, value
        got = run(*bad)
        for x, y in zip(got, base):
            assert torch.equal(x[keep], y[keep])
        assert not got[0][165].isfinite().any()
        assert torch.equal(got[0][150:160], base[0][150:160])  # (rows before it do not see it)


def test_strides_and_one_buffer(kernels_only):
    starts = torch.tensor([0, 60, 100], device=dev())
    buf = _rand(100, 3, 4, 64)
    q, k, v = buf.unbind(1)
    do = _rand(100, 4, 64, seed=9)

    def run(*t, do=do, starts=starts):
        t = [x.detach().requires_grad_(True) for x in t]
        o = F.packed_attention(*t, starts, window=30, sinks=2)
        return o, *torch.autograd.grad(o, t, do)

    plain = run(*(t.contiguous() for t in (q, k, v)))
    off = torch.empty(q.numel() + 3, dtype=torch.bfloat16, device=dev())[3:].view(q.shape).copy_(q)
    heads_first = k.transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.zeros(100, 4, 68, dtype=torch.bfloat16, device=dev())
    wide[..., :64] = v
    strided = torch.stack((starts, starts + 7), 1)[:, 0]
    for t, more in (((q, k, v), {}), ((off, heads_first, wide[..., :64]), {}), ((q, k, v), dict(starts=strided)),
                    ((q, k, v), dict(do=do.transpose(0, 1).contiguous().transpose(0, 1)))):
        for x, y in zip(run(*t, **more), plain):
            assert torch.equal(x, y)
    # one head of k and v for all, as a broadcast
    kk, vv = (t[:, :1].detach().clone().requires_grad_(True) for t in (k, v))
    o = F.packed_attention(q, kk.expand(100, 4, 64), vv.expand(100, 4, 64), starts)
    got = torch.autograd.grad(o, (kk, vv), do)
    full = [t[:, :1].expand(100, 4, 64).contiguous().requires_grad_(True) for t in (k, v)]
    for x, y in zip(got, torch.autograd.grad(F.packed_attention(q, *full, starts), full, do)):
        assert torch.equal(x, y.sum(1, keepdim=True))
    # some of the gradients
    for i in range(3):
        t = [x.detach().requires_grad_(i == j) for j, x in enumerate((q, k, v))]
        (g,) = torch.autograd.grad(F.packed_attention(*t, starts, window=30, sinks=2), t[i], do)
        assert torch.equal(g, plain[1 + i])


def test_starts_written_after_the_forward(kernels_only):
    """The backward goes by the forward's table."""
    q, k, v, do = _inputs(200, 2, 2, 64)
    starts = torch.tensor([0, 50, 200], device=dev())
    expect = torch.autograd.grad(F.packed_attention(q, k, v, starts), (q, k, v), do)
    o = F.packed_attention(q, k, v, starts)
    starts.fill_(7)
    for x, y in zip(torch.autograd.grad(o, (q, k, v), do), expect):
        assert torch.equal(x, y)


def test_starts_out_of_order(kernels_only):
    q, k, v, do = _inputs(300, 2, 1, 64)
    for given, meant in (([-3, 170, 20, 10 ** 9], [0, 170, 170, 300]), ([140, 10, 200], [140, 140, 200])):
        o = F.packed_attention(q, k, v, torch.tensor(given, device=dev()))
        _check((o, *torch.autograd.grad(o, (q, k, v), do)), q, k, v, do, meant, None, 0)


def test_many_sequences(kernels_only):
    """More than the plan's workgroup has threads, most of them of a row or none."""
    g = torch.Generator().manual_seed(5)
    lengths = torch.randint(0, 3, (5000,), generator=g)
    lengths[2500] = 700
    starts = torch.cat((torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)))
    rows = int(starts[-1]) + 5
    q, k, v, do = _inputs(rows, 2, 1, 64)
    o = F.packed_attention(q, k, v, starts.to(dev()), window=50, sinks=1)
    got = (o, *torch.autograd.grad(o, (q, k, v), do))
    few = [0, 1, 2, 2500, 4999]
    for s in few:
        a, b = int(starts[s]), int(starts[s + 1])
        if a == b:
            continue
        padded = [t.detach()[a:b].transpose(0, 1).unsqueeze(0) for t in (q, k, v, do)]
        refs, tols = _reference(*padded, 50, 1, None, 0.125)
        for x, r, t in zip(got, refs, tols):
            _within(x.detach()[a:b].transpose(0, 1).unsqueeze(0).cpu(), r, t, s)
    # sequences of one row: o is v
    ones = starts[:-1][lengths == 1].to(dev())
    assert torch.equal(o[ones], v[ones].expand(-1, 2, -1))
    assert not got[0][-5:].any() and not got[2][-5:].any()


def test_another_stream_and_graphs(kernels_only):
    q, k, v, do = _inputs(500, 4, 2, 64)
    starts = torch.tensor([0, 100, 130, 490], device=dev())

    def step():
        o = F.packed_attention(q, k, v, starts, window=70, sinks=2)
        return [o, *torch.autograd.grad(o, (q, k, v), do)]

    ref = [r.detach().clone() for r in step()]
    other = torch.tensor([0, 300, 301, 450], device=dev())
    first = starts.clone()
    starts.copy_(other)
    ref2 = [r.detach().clone() for r in step()]
    starts.copy_(first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            out = step()
    torch.cuda.current_stream().wait_stream(s)
    for a, r in zip(out, ref):
        assert torch.equal(a, r)
    del out
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    # replayed for other sequences of the same number and rows
    for given, expect in ((first, ref), (other, ref2), (first, ref)):
        starts.copy_(given)
        for a in out:
            a.detach().zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, r in zip(out, expect):
            assert torch.equal(a, r)
        step()


def test_routes():
    """What the kernels do not take is torch's, with the same results within bf16; a recorded backward."""
    starts = torch.tensor([0, 10, 40], device=dev())
    q, k, v, do = _inputs(40, 2, 2, 64)
    o = F.packed_attention(q, k, v, starts, window=9)
    for t in (torch.float32, torch.float64):
        y = F.packed_attention(*(x.detach().to(t) for x in (q, k, v)), starts, window=9)
        assert y.dtype == t and (y - o).abs().max() <= 4 * 2.0 ** -8 * v.abs().max()
    assert F.packed_attention(*(_rand(5, 1, 12, seed=s) for s in range(3)), starts).shape == (5, 1, 12)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        F.packed_attention(q, k, v, starts)
    first = torch.autograd.grad(o, (q, k, v), do)
    recorded = torch.autograd.grad(F.packed_attention(q, k, v, starts, window=9), (q, k, v), do, create_graph=True)
    for x, y in zip(first, recorded):
        assert (x.double() - y.double()).norm() <= 4 * 2.0 ** -8 * y.double().norm()
    torch.autograd.grad(sum(x.float().sum() for x in recorded), (q, k, v))


@pytest.mark.parametrize("scale", [0.01, 3.0])
def test_sharp_and_flat(kernels_only, scale):
    q, k, v, do = (_rand(400, 2, 64, seed=s, scale=1.5) for s in range(4))
    q, k, v = (t.requires_grad_(True) for t in (q, k, v))
    starts = [0, 200, 330, 400]
    o = F.packed_attention(q, k, v, torch.tensor(starts, device=dev()), window=150, sinks=2, scale=scale)
    _check((o, *torch.autograd.grad(o, (q, k, v), do)), q, k, v, do, starts, 150, 2, scale)


def test_against_differences():
    """The gradients agree with differences of the float64 definition's loss along random directions."""
    q, k, v, do = _inputs(150, 4, 2, 64)
    starts = torch.tensor([0, 47, 150], device=dev())
    o = F.packed_attention(q, k, v, starts, window=40, sinks=2)
    grads = torch.autograd.grad(o, (q, k, v), do)
    wide = [t.detach().double() for t in (q, k, v)]
    loss = lambda *t: (F.packed_attention(*t, starts, window=40, sinks=2) * do.double()).sum()
    for i, g in enumerate(grads):
        d = _rand(*g.shape, seed=20 + i).double()
        h = 1e-4
        up, down = ([w + s * h * d if j == i else w for j, w in enumerate(wide)] for s in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * h)
        # each element is off by the rounding of the operands and of itself: 2^-6 of the terms' sum
        assert abs((g.double() * d).sum() - slope) <= 2.0 ** -6 * (g.double() * d).abs().sum()


def test_offsets_past_32_bits(kernels_only):
    """Rows 2^23 elements apart: the last ones past 2^31."""
    if torch.cuda.get_device_properties(0).total_memory < 32 << 30:
        pytest.skip("memory")
    rows, apart, hd = 300, 1 << 23, 64
    buf = torch.empty(rows * apart, dtype=torch.bfloat16, device=dev())
    t = []
    for i, heads in enumerate((2, 1, 1)):
        x = buf[256 * i:].as_strided((rows, heads, hd), (apart, hd, 1))
        t.append(x.copy_(_rand(rows, heads, hd, seed=i)))
    starts, do = torch.tensor([0, 20, 290], device=dev()), _rand(rows, 2, hd, seed=9)

    def run(*t):
        t = [x.detach().requires_grad_(True) for x in t]
        o = F.packed_attention(*t, starts, window=100, sinks=2)
        return o, *torch.autograd.grad(o, t, do)

    for x, y in zip(run(*t), run(*(x.contiguous() for x in t))):
        assert torch.equal(x, y)


def test_more_heads_and_sequences_than_one_launch_finds_itself(kernels_only):
    """On both sides of the rule for a forward without the table: the same bits."""
    for n, heads in ((F.OWN_SEQUENCES, 2), (F.OWN_SEQUENCES + 1, 2), (3, 64), (3, 200)):
        rows = 10 * n + 3
        starts = [1 + 10 * i for i in range(n + 1)]
        q, k, v, do = _inputs(rows, heads, 2, 64)
        table = F.packed_wants_table(n, rows, heads)
        assert table == (n > F.OWN_SEQUENCES or heads == 200)
        at = torch.tensor(starts, device=dev())
        plain = F.packed_attention(q.detach(), k.detach(), v.detach(), at, window=7)
        o = F.packed_attention(q, k, v, at, window=7)
        assert torch.equal(plain, o)
        if n == 3:
            _check((o,), q, k, v, do, starts, 7, 0)


def test_two_streams_at_once(kernels_only):
    """Calls that run beside each other share nothing."""
    starts = [torch.tensor(s, device=dev()) for s in ([0, 300, 700], [100, 200, 650])]
    t = [_inputs(700, 8, 2, 64, seed=10 * i) for i in range(2)]

    def step(i):
        q, k, v, do = t[i]
        o = F.packed_attention(q, k, v, starts[i], window=150, sinks=3)
        return o, *torch.autograd.grad(o, (q, k, v), do)

    expect = [[x.detach().clone() for x in step(i)] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = step(i)
    torch.cuda.synchronize()
    for a, b in zip(got, expect):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
