"""Which form of rotary positions, attention and distillation answers, and what its backward
keeps, without a GPU: the kernels' routes run on CPU tensors with launches that are noted
instead of made, so a kernel's results are unwritten memory and only the rest is looked at."""
import math
import struct

import pytest

torch = pytest.importorskip("torch")
F = pytest.importorskip("paper_2410_15352_amd.functional")

bf16, f32, f64 = torch.bfloat16, torch.float32, torch.float64


def _rand(*shape, seed=0, dtype=bf16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed + sum(shape))).to(dtype)


@pytest.fixture
def launches(monkeypatch):
    """Entry points called, in order."""
    names = []
    monkeypatch.setattr(F, "_here", F._plain)
    monkeypatch.setattr(F, "_stream", lambda t: 0)
    monkeypatch.setattr(F.ops, "_call", lambda name, *args: names.append(name))
    monkeypatch.setattr(F.ops, "_companion", lambda t, dtype, count: (
        t.dtype == dtype and t.numel() == count and F._plain(t) and t.is_contiguous()))
    monkeypatch.setattr(F, "_attn_scratch", lambda block: 0)
    return names


# --------------------- saved tensors from a hook -----------------------------

def _attention_with_hook(unpack):
    q, k, v = (_rand(2, 2, 5, 8, seed=s).requires_grad_() for s in (1, 2, 3))
    do = _rand(2, 2, 5, 8, seed=4)
    lengths = torch.tensor([5, 3], dtype=torch.int32)
    rule = dict(window=3, sinks=1, lengths=lengths)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        o = F.window_attention(q, k, v, **rule)
    grads = torch.autograd.grad(o, (q, k, v), do)
    wide = [t.detach().to(f64).requires_grad_() for t in (q, k, v)]
    expect = torch.autograd.grad(F.window_attention(*wide, **rule), wide, do.to(f64))
    return grads, expect


def test_attention_saved_tensors_as_they_were(launches):
    _attention_with_hook(lambda t: t)
    assert launches == ["compact_attention_fwd", "compact_attention_bwd"]


@pytest.mark.parametrize("unpack", [
    lambda t: t.long() if t.dtype == torch.int32 else t,           # lengths of another type
    lambda t: torch.stack((t, t), 1)[:, 0] if t.dtype == torch.int32 else t,  # not dense
    lambda t: t.float() if t.dtype == bf16 else t])
def test_attention_saved_tensors_changed_by_a_hook(launches, unpack):
    """The kernel would read lengths as int32 from a pointer of the GPU's: it must not run on others."""
    grads, expect = _attention_with_hook(unpack)
    assert launches == ["compact_attention_fwd"]
    for g, e in zip(grads, expect):
        assert g.dtype == bf16 and (g.double() - e).abs().max() <= 2.0 ** -7 * e.abs().max()


def _distill_with_hook(unpack, dtype=bf16):
    x, top = _rand(4, 24, seed=1, dtype=dtype).requires_grad_(), _rand(4, 3, seed=2)
    ids, targets = torch.arange(12).view(4, 3), torch.tensor([0, -100, 5, 23])
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        loss = F._DistillFn.apply(x, top, ids, targets, 2.0, 0.5)
    (g,) = torch.autograd.grad(loss, x, torch.tensor(3.0))
    wide = x.detach().double().requires_grad_()
    (e,) = torch.autograd.grad(F.distill_loss(wide, top.double(), ids, targets=targets, temperature=2.0, weight=0.5), wide,
                               torch.tensor(3.0, dtype=f64))
    return g, e


def test_distill_saved_tensors_as_they_were(launches):
    _distill_with_hook(lambda t: t)
    assert launches == ["compact_distill"] * 2


@pytest.mark.parametrize("unpack", [
    lambda t: t.float() if t.shape == (4, 24) else t,               # logits of a wider type than the gradient's buffer
    lambda t: t.int() if t.shape == (4,) else t,                    # targets read as int64
    lambda t: torch.stack((t, t), -1)[..., 0] if t.shape == (4,) else t])
def test_distill_saved_tensors_changed_by_a_hook(launches, unpack):
    """The gradient's buffer is of the forward's type and size: no kernel writes it for others."""
    g, e = _distill_with_hook(unpack)
    assert launches == ["compact_distill"]
    assert g.dtype in (bf16, f32) and (g.double() - e).abs().max() <= 2.0 ** -7 * e.abs().max()


# ------------------------------- autocast ------------------------------------

def test_attention_under_autocast_stays_in_32_bits():
    """The torch expressions' products are fp32 ones, forward and backward, whatever autocast makes of products."""
    t = [_rand(2, 4, 9, 8, seed=s, dtype=f32).requires_grad_() for s in (1, 2, 3)]
    do = _rand(2, 4, 9, 8, seed=4, dtype=f32)
    plain = F.window_attention(*t, window=4, sinks=1)
    with torch.autocast("cpu", dtype=bf16):
        o = F.window_attention(*t, window=4, sinks=1)
    assert o.dtype == f32 and torch.equal(o, plain)
    for a, b in zip(torch.autograd.grad(o, t, do), torch.autograd.grad(plain, t, do)):
        assert torch.equal(a, b)


def test_attention_of_tensors_without_storage():
    q = torch.empty(1, 2, 5, 8, device="meta")
    assert F.window_attention(q, q, q, window=3).shape == q.shape


# ------------------------------- rotary --------------------------------------

@pytest.fixture
def turned_by_kernels(monkeypatch):
    """Rotary's kernel route, its launches made by the torch expressions."""
    monkeypatch.setattr(F, "_here", F._plain)
    monkeypatch.setattr(F, "_rotary_apply", lambda rope, positions, inverse, *t: [
        y for y in F._rotary_torch(rope, positions, bool(inverse), *t) if y is not None])

    def call(rope, positions, inverse, x, fields, count):  # in place, of qkv's q and k
        calls.append((positions, inverse))
    calls = []
    monkeypatch.setattr(F, "_rotary_call", call)
    return calls


def _rotary_step(kind, positions):
    """(gradient, its inputs) of one rotation with the given positions, as a function that runs the backward."""
    rope = F.Rotary(8)
    if kind == "in place":
        qkv = _rand(2, 4, 3, 2, 8, seed=1, dtype=f32).requires_grad_()
        out = F.rotary_split_qkv(qkv * 1, rope, positions=positions)
        return lambda: torch.autograd.grad(sum(t.sum() for t in out), qkv)
    q, k = (_rand(2, 4, 2, 8, seed=s, dtype=f32).requires_grad_() for s in (1, 2))
    if kind == "q":
        y = rope(q, positions=positions)
        return lambda: torch.autograd.grad(y, q, torch.ones_like(y))
    y = rope(q, k, positions=positions)
    return lambda: torch.autograd.grad(y, (q, k), [torch.ones_like(x) for x in y])


@pytest.mark.parametrize("kind", ["q", "q and k", "in place"])
def test_rotary_positions_written_before_the_backward(turned_by_kernels, kind):
    """A buffer of positions that moved on: the angles of the forward are gone, and autograd says so."""
    positions = torch.arange(4)
    back = _rotary_step(kind, positions)
    back()
    back = _rotary_step(kind, positions)
    positions += 4
    with pytest.raises(RuntimeError, match="inplace operation"):
        back()


@pytest.mark.parametrize("kind", ["q", "q and k", "in place"])
def test_rotary_positions_through_saved_tensor_hooks(turned_by_kernels, kind):
    """Positions that come back in another type turn back by the same angles."""
    positions = torch.tensor([[3, 1, 4, 1], [5, 9, 2, 6]])
    plain = _rotary_step(kind, positions)()
    if kind == "in place":
        assert torch.equal(turned_by_kernels[-1][0], positions)
    packed = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: packed.append(t) or t.to(torch.int16), lambda t: t):
        back = _rotary_step(kind, positions)
    assert any(t is positions or torch.equal(t, positions) for t in packed)
    for a, b in zip(back(), plain):
        assert kind == "in place" or torch.equal(a, b)
    if kind == "in place":
        assert turned_by_kernels[-1][0].dtype == positions.dtype and torch.equal(turned_by_kernels[-1][0], positions)


# --------------------- recorded backwards of attention -----------------------

RULE = dict(window=3, sinks=1)


def _recorded(make, dtype):
    """First and second derivatives by x of attention whose q, k and v are make(x); bf16 takes the kernels' route."""
    x = _rand(3, 1, 2, 6, 8, seed=5).to(dtype).requires_grad_()
    do = _rand(1, 2, 6, 8, seed=6).to(dtype)
    q, k, v = make(x)
    o = F.window_attention(q, k, v, **RULE)
    leaves = [x, *(t for t in (q, k, v) if t is not x)]
    first = torch.autograd.grad(o, leaves, do, create_graph=True)
    (second,) = torch.autograd.grad(first[0].double().square().sum(), x)
    return [*first, second]


DEPENDENT = {
    "separate": lambda x: (x[0], x[1], x[2]),
    "v is k": lambda x: (lambda k: (x[0], k, k))(x[1] * 1),
    "v from k": lambda x: (lambda k: (x[0], k, 2 * k))(x[1] * 1),
    "q, k and v are one": lambda x: (lambda t: (t, t, t))(x[0] * 1),
    "q from v from k": lambda x: (lambda k: (lambda v: (v + x[0], k, v))(k * x[2]))(x[1] * 1),
}


@pytest.mark.parametrize("name", list(DEPENDENT))
def test_recorded_backward_of_inputs_that_depend_on_one_another(launches, name):
    got, ref = _recorded(DEPENDENT[name], bf16), _recorded(DEPENDENT[name], f64)
    assert launches == ["compact_attention_fwd"]
    for a, b in zip(got, ref):
        # bf16 results of a few roundings each
        assert (a.double() - b).norm() <= 2.0 ** -5 * b.norm()


COPIED = {
    "q off the 16-byte boundary": lambda x: (torch.nn.functional.pad(x[0].reshape(-1), (1, 0))[1:].view(x[0].shape), x[1], x[2]),
    "q's rows 12 apart": lambda x: (torch.nn.functional.pad(x[0], (0, 4))[..., :8], x[1], x[2]),
    "k's last dimension strided": lambda x: (x[0], x[1].transpose(2, 3).contiguous().transpose(2, 3), x[2]),
    "v's rows on one another": lambda x: (x[0], x[1], x[2].reshape(-1).as_strided((1, 2, 6, 8), (96, 48, 4, 1))),
}


@pytest.mark.parametrize("name", list(COPIED))
def test_recorded_backward_of_inputs_that_are_copied(launches, name):
    """The kernels read a dense, aligned copy: its history reaches the second derivatives."""
    assert any(F._attn_tensor(t)[0] is not t for t in COPIED[name](_rand(3, 1, 2, 6, 8)))
    got, ref = _recorded(COPIED[name], bf16), _recorded(COPIED[name], f64)
    assert launches == ["compact_attention_fwd"]
    for a, b in zip(got, ref):
        assert (a.double() - b).norm() <= 2.0 ** -5 * b.norm()


# ------------------------- a Rotary's frequencies -----------------------------

def _fake_rotation(rope):
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        assert rope(torch.zeros(1, 2, 1, 8)).shape == (1, 2, 1, 8)


def _traced_rotation(rope):
    from torch.fx.experimental.proxy_tensor import make_fx
    x = _rand(1, 2, 1, 8, dtype=f32)
    assert torch.equal(make_fx(rope, tracing_mode="fake")(x)(x), F.Rotary(8)(x))


FIRST_USES = {
    "func.grad": lambda rope: torch.func.grad(lambda q: rope(q).sum())(_rand(1, 2, 1, 8, dtype=f32)),
    "vmap": lambda rope: torch.func.vmap(rope)(_rand(3, 1, 2, 1, 8, dtype=f32)),
    "fake tensors": _fake_rotation,
    "make_fx": _traced_rotation,
    "inference": lambda rope: torch.inference_mode()(rope)(_rand(1, 2, 1, 8, dtype=f32)),
    "meta": lambda rope: rope(torch.zeros(1, 2, 1, 8, device="meta")),
}


@pytest.mark.parametrize("name", list(FIRST_USES))
def test_rotary_first_used_under_a_transform(name):
    """What a transform makes of the frequencies is not kept for later calls."""
    rope = F.Rotary(8)
    # (a device's copy as on a GPU: none yet)
    rope._turns.clear()
    FIRST_USES[name](rope)
    turns = rope.turns(torch.device("cpu"))
    assert type(turns) is torch.Tensor and turns.data_ptr() != 0 and not turns.is_inference()
    assert torch.equal(turns, F.Rotary(8).turns(torch.device("cpu")))
    x = _rand(1, 2, 1, 8, dtype=f32)
    assert torch.equal(rope(x), F.Rotary(8)(x))


def test_rotary_made_under_another_device():
    with torch.device("meta"):
        rope = F.Rotary(8)
    x = _rand(1, 2, 1, 8, dtype=f32)
    assert torch.equal(rope(x), F.Rotary(8)(x))


def test_rotary_copied_and_saved():
    import copy
    import pickle
    rope = F.Rotary(8, scaling="linear", factor=2.0)
    x = _rand(1, 2, 1, 8, dtype=f32)
    for other in (copy.deepcopy(rope), pickle.loads(pickle.dumps(rope))):
        assert torch.equal(other(x), rope(x))


# --------------------------- sizes of a call's plan ---------------------------

def _scratch_bytes(b, heads, kv, l, hd, window, sinks):
    """The backward's scratch for sums in parts, as the library plans it (no launch)."""
    lib = pytest.importorskip("paper_2410_15352_amd._lib").load()
    fn = lib.compact_attention_bwd_scratch
    fn.restype, fn.argtypes = F._i64, [F._block]
    rows = (l * hd, hd, hd)
    floats = fn(F._attn_pack(*(0,) * 7, *rows, *rows, *rows, *rows, b, heads, kv, l, l, hd,
                             F.NO_WINDOW if window is None else window, sinks, 1.0, 0, 0, 0, 0))
    return 4 * floats


@pytest.mark.parametrize("b,heads,kv,l,hd", [(4, 16, 16, 16384, 64), (1, 16, 16, 16384, 64), (1, 16, 4, 16384, 128),
                                             (1, 1, 1, 65536, 64), (2, 4, 1, 70000, 96), (64, 8, 8, 4096, 32)])
@pytest.mark.parametrize("window", [128, 1024])
def test_attention_scratch_is_bounded(b, heads, kv, l, hd, window):
    """However many sinks: two slots and the window's own of dk and dv in fp32 for each sink (6 times
    k's and v's bytes if all are sinks), or those of 1024 workgroups of 128 keys."""
    for sinks in (1, 4, 64, 1000, 4096, l // 2, l - window - 1):
        assert 0 <= _scratch_bytes(b, heads, kv, l, hd, window, sinks) <= (
            6 * 4 * b * kv * l * hd + 2 * 4 * 2 * hd * 1024 * 128)


def test_attention_of_sinks_that_reach_the_window(launches, monkeypatch):
    """Window and sinks that cover a sequence are no window: no sums in parts for the sinks."""
    blocks = []
    monkeypatch.setattr(F.ops, "_call", lambda name, block, stream: blocks.append(block))
    q, k, v = (_rand(1, 2, 100, 8, seed=s) for s in (1, 2, 3))
    for window, sinks, expect in ((30, 70, (F.NO_WINDOW, 0)), (30, 1000, (F.NO_WINDOW, 0)), (30, 69, (30, 69)), (None, 5, (F.NO_WINDOW, 0))):
        F.window_attention(q, k, v, window=window, sinks=sinks)
        fields = struct.unpack("@" + F._ATTN, blocks[-1])
        assert fields[25] == expect[0] and (window is None or fields[26] == expect[1]), (window, sinks)


def _limits():
    """Sizes around the limits of a call's launches: (b, heads, kv, lq, lk, hd)."""
    for kv in (1, 8, 128):
        for G in (1, 16, 1 << 12, 1 << 17):
            for lq in (1, 31, 32, 33, 128, 4096):
                for rows in (1 << 18, 1 << 21, 1 << 22, 1 << 23, (1 << 24) - 1, 1 << 24, 1 << 28, (1 << 29) - 64):
                    for b in {max(1, rows // (kv * G * lq)), max(1, rows // (kv * G * lq) - 1), max(1, rows // (kv * G))}:
                        for lk in (1, 32, 4096, 70000):
                            for hd in (8, 128):
                                yield b, kv * G, kv, lq, lk, hd


def test_attention_calls_that_are_taken_are_launched(monkeypatch):
    """What _attention_usable lets through, the entry points take: their limits on a launch's grid."""
    monkeypatch.setattr(F, "_here", lambda t: True)
    taken = 0
    for b, heads, kv, lq, lk, hd in _limits():
        q, k = (torch.empty(1, dtype=bf16).expand(b, n, l, hd) for n, l in ((heads, lq), (kv, lk)))
        for window, sinks in ((F.NO_WINDOW, 0), (7, 3), (7, max(0, lk - 8))):
            if F._attention_usable(q, k, k, False):
                taken += 1
                rows = b * heads * lq
                splits = F.attention_splits(b, heads, kv, lq, lk, window, sinks)
                few = lq <= F.FEW_ROWS
                assert 0 <= splits <= 4096
                if splits > 0:
                    assert rows < 1 << 24 and b * heads * -(-lq // 128) * splits < 1 << 31
                    assert not few or b * kv <= 65535 and -(-(heads // kv * lq) // 32) <= 65535
                if splits == 0 or not few:
                    assert b * heads * -(-lq // 128) * max(1, splits) * 256 < 1 << 32
            if F._attention_usable(q, k, k, True):
                assert _scratch_bytes_of(b, heads, kv, lq, lk, hd, window, sinks) >= 0, (b, heads, kv, lq, lk, hd, window, sinks)
    assert taken > 500


def _scratch_bytes_of(b, heads, kv, lq, lk, hd, window, sinks):
    lib = pytest.importorskip("paper_2410_15352_amd._lib").load()
    fn = lib.compact_attention_bwd_scratch
    fn.restype, fn.argtypes = F._i64, [F._block]
    rows = (lk * hd, hd, hd)
    return fn(F._attn_pack(*(0,) * 7, *rows, *rows, *rows, *rows, b, heads, kv, lq, lk, hd, window, sinks, 1.0, 0, 0, 0, 0))


def test_attention_plans_that_pass_a_launch_are_refused():
    """128 columns of dk and dv: 512 threads for 128 keys."""
    assert _scratch_bytes_of(1 << 20, 8, 8, 1, 32, 128, F.NO_WINDOW, 0) < 0
    assert _scratch_bytes_of(1 << 20, 8, 8, 1, 32, 64, F.NO_WINDOW, 0) >= 0
    assert _scratch_bytes_of(1 << 18, 8, 8, 1, 32, 128, F.NO_WINDOW, 0) >= 0


# --------------------------- the block's projection ---------------------------

def _block():
    blk = pytest.importorskip("paper_2410_15352_amd.block")
    torch.manual_seed(0)
    return blk.LlamaBlock(32, 2, 32, device="cpu", rope=F.Rotary(16), window=4)


WATCHED = {
    "forward hook": lambda b: b.qkv.register_forward_hook(lambda m, x, y: None),
    "backward hook": lambda b: b.qkv.register_full_backward_hook(lambda m, x, y: None),
    "hook of all modules": lambda b: torch.nn.modules.module.register_module_forward_hook(lambda m, x, y: None),
    "forward replaced": lambda b: setattr(b.qkv, "forward", type(b.qkv).forward.__get__(b.qkv)),
    "module replaced": lambda b: setattr(b, "qkv", torch.nn.Sequential(b.qkv)),
}


@pytest.mark.parametrize("name", list(WATCHED))
def test_projection_whose_output_may_be_kept_is_not_rotated_in_place(turned_by_kernels, monkeypatch, name):
    in_place = []
    monkeypatch.setattr(F, "_rotary_call", lambda *a: in_place.append(a))
    monkeypatch.setattr(F, "_attention_usable", lambda *a: False)
    b, x = _block(), _rand(1, 8, 32, seed=1)
    b(x)
    assert len(in_place) == 1
    handle = WATCHED[name](b)
    try:
        y = b(x)
    finally:
        if handle is not None:
            handle.remove()
    assert len(in_place) == 1
    # (rotated all the same)
    monkeypatch.setattr(F, "_here", lambda t: False)
    assert torch.equal(y, b(x))


# ------------------------------- no keys --------------------------------------

@pytest.mark.parametrize("heads,kv", [(2, 2), (4, 2)])
def test_attention_over_no_keys(heads, kv):
    """Zeros whatever q holds, and gradients of every input: zeros, and empty ones."""
    q = torch.full((2, heads, 3, 8), math.nan, dtype=f64).requires_grad_()
    k, v = (torch.empty(2, kv, 0, 8, dtype=f64).requires_grad_() for _ in range(2))
    for lengths in (None, torch.zeros(2, dtype=torch.int64)):
        o = F.window_attention(q, k, v, window=4, lengths=lengths)
        assert torch.equal(o, torch.zeros_like(o))
        dq, dk, dv = torch.autograd.grad(o, (q, k, v), torch.ones_like(o))
        assert torch.equal(dq, torch.zeros_like(dq)) and dk.shape == k.shape and dv.shape == v.shape


# ------------------------------- refusals -------------------------------------

def _attend(**change):
    t = dict(q=torch.zeros(2, 2, 3, 8), k=torch.zeros(2, 2, 4, 8), v=torch.zeros(2, 2, 4, 8))
    return F.window_attention(**{**t, **change})


def _distill(**change):
    t = dict(logits=torch.zeros(2, 4), top_logits=torch.zeros(2, 1), top_ids=torch.zeros(2, 1).long())
    return F.distill_loss(**{**t, **change})


@pytest.mark.parametrize("call", [
    lambda: _attend(window=2.5), lambda: _attend(window=2, sinks=1.0), lambda: _attend(window="4"), lambda: _attend(lengths=[4, 4]),
    lambda: _attend(q=[1]), lambda: _distill(targets=[0, 1], weight=0.5), lambda: _distill(top_ids=[[0], [0]]),
    lambda: F.Rotary(8)([1.0])])
def test_arguments_of_other_kinds_are_refused(call):
    with pytest.raises(TypeError):
        call()


@pytest.mark.parametrize("call", [
    lambda: _attend(q=torch.zeros(2, 2, 3, 0), k=torch.zeros(2, 2, 4, 0), v=torch.zeros(2, 2, 4, 0)),
    lambda: _distill(logits=torch.zeros(2, 0)), lambda: F.Rotary(8, factor=math.inf), lambda: F.Rotary(8, base=math.inf),
    lambda: F.Rotary(8, scaling="parts", original_length=math.inf), lambda: F.Rotary(8, high=math.inf),
    lambda: F.Rotary(8)(torch.zeros(1, 2, 1, 8), positions=1 << 63), lambda: F.Rotary(8)(torch.zeros(1, 2, 1, 8), positions=-1 << 70)])
def test_values_past_what_is_defined_are_refused(call):
    with pytest.raises(ValueError):
        call()


def test_arguments_that_stay_allowed():
    import numpy as np
    o = _attend(window=np.int64(2), sinks=np.int32(1))
    assert o.shape == (2, 2, 3, 8)
    assert F.Rotary(8)(torch.zeros(1, 2, 1, 8), positions=1 << 40).shape == (1, 2, 1, 8)
    assert _distill(logits=torch.zeros(0, 4), top_logits=torch.zeros(0, 1), top_ids=torch.zeros(0, 1).long()).isnan()


def test_factors_past_fp32_are_the_torch_expressions(launches):
    """The kernels hold scale and temperature in fp32; others are not theirs."""
    q, k, v = (_rand(1, 2, 5, 8, seed=s) for s in (1, 2, 3))
    for scale in (1e-45, 1e-60, 1e40):
        assert F.window_attention(q, k, v, scale=scale).shape == q.shape
    x, top, ids = _rand(2, 8, dtype=f32), _rand(2, 2, dtype=f32), torch.tensor([[0, 1], [2, 3]])
    assert not F._distill_taken(1e-45) and not F._distill_taken(1e40) and F._distill_taken(2.0)
    assert F.distill_loss(x, top, ids, temperature=1e40).dtype == f32
    assert launches == []
    F.window_attention(q, k, v, scale=1e-3)
    assert launches == ["compact_attention_fwd"]
