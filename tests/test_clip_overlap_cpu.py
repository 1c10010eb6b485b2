"""Clipping tensors that share memory: the same elements, in whatever shape or order, count once, a part of
them shared is refused, whichever form answers; slices beside one another are neither."""
import math
import random

import pytest

torch = pytest.importorskip("torch")
FT = pytest.importorskip("paper_2410_15352_amd.finetune")

f16, bf16, f32, f64 = torch.float16, torch.bfloat16, torch.float32, torch.float64


@pytest.mark.parametrize("again", [
    lambda x: x.view(4, 6), lambda x: x.view(4, 6).t(), lambda x: x.view(2, 3, 4).permute(2, 0, 1), lambda x: x.view(1, 24, 1),
    lambda x: x[:]], ids=["shape", "transposed", "permuted", "ones", "view"])
@pytest.mark.parametrize("dtype", [f16, bf16, f32, f64])
def test_the_same_elements_count_once(again, dtype):
    x = torch.full((24,), 2.0, dtype=dtype)
    norm = 2 * 24 ** 0.5
    assert math.isclose(float(FT.clip_grad_norm([x, again(x)])), norm, rel_tol=1e-6)
    assert math.isclose(float(FT.clip_grad_norm([again(x), x], 1.0)), norm, rel_tol=1e-6)
    # scaled once: its rounding, at most half a step
    assert ((x.double() - 24 ** -0.5).abs() <= (torch.finfo(dtype).eps / 2 + 2e-7) * 24 ** -0.5).all()


def test_the_same_slices_count_once():
    x = torch.ones(5, 8)
    a = x[:, 2:6]
    assert math.isclose(float(FT.clip_grad_norm([a, a.t(), x[:, :2], x[:, 6:], a], 1.0)), 40 ** 0.5, rel_tol=1e-6)
    assert (x - 40 ** -0.5).abs().max() < 1e-6


OVERLAPS = {
    "ends": lambda b: (b[:60], b[40:]), "inside": lambda b: (b, b[10:20]), "columns": lambda b: (b.view(10, 10)[:, :6], b.view(10, 10)[:, 4:]),
    "a row of columns": lambda b: (b.view(10, 10)[:, 3], b.view(10, 10)[4]), "every second": lambda b: (b[::2], b[::3]),
    "rows and columns": lambda b: (b.view(10, 10)[2:5, 2:5], b.view(10, 10)[4:, 4:]), "another type": lambda b: (b, b.view(torch.int32).view(f32)[:1]),
    "halves": lambda b: (b, b.view(f16))}


@pytest.mark.parametrize("which", list(OVERLAPS))
@pytest.mark.parametrize("bound", [None, 1.0])
def test_a_part_shared_is_refused(which, bound):
    b = torch.ones(100)
    with pytest.raises(ValueError, match="overlap"):
        FT.clip_grad_norm([torch.ones(3, dtype=f64), *OVERLAPS[which](b)], bound)
    assert (b == 1).all()


APART = {
    "columns": lambda b: (b.view(10, 10)[:, :6], b.view(10, 10)[:, 6:]), "odd and even": lambda b: (b[::2], b[1::2]),
    "quarters": lambda b: (b.view(10, 10)[:4, :4], b.view(10, 10)[:4, 4:], b.view(10, 10)[4:, :4], b.view(10, 10)[4:, 4:]),
    "heads": lambda b: (b.view(5, 4, 5)[:, :2], b.view(5, 4, 5)[:, 2:, :3], b.view(5, 4, 5)[:, 2:, 3:]),
    "diagonal beside": lambda b: (b.view(10, 10).diagonal(), b[1::11])}


@pytest.mark.parametrize("which", list(APART))
def test_slices_beside_one_another(which):
    b = torch.ones(100)
    t = APART[which](b)
    n = sum(x.numel() for x in t)
    assert math.isclose(float(FT.clip_grad_norm(t, 1.0)), n ** 0.5, rel_tol=1e-6)
    assert all((x - n ** -0.5).abs().max() < 1e-6 for x in t) and int((b != 1).sum()) == n


def test_against_every_byte():
    """Random strided views of one buffer, against the sets of their bytes."""
    rng = random.Random(3)
    buf = torch.zeros(4096, dtype=torch.uint8)
    shared = 0
    for _ in range(3000):
        views, sets = [], []
        for _ in range(2):
            dtype = rng.choice((f16, f32))
            size = torch.empty((), dtype=dtype).element_size()
            base = buf.view(dtype)
            shape = [rng.randint(1, 4) for _ in range(rng.randint(0, 3))]
            stride = [rng.choice((0, 1, 1, 2, 3, 4, 6, 8, 12)) for _ in shape]
            at = rng.randint(0, 40)
            views.append(base.as_strided(shape, stride, at))
            places = [at]
            for n, s in zip(shape, stride):
                places = [p + i * s for p in places for i in range(n)]
            sets.append({p * size + k for p in places for k in range(size)})
        same = views[0].dtype == views[1].dtype and sets[0] == sets[1]
        meet = bool(sets[0] & sets[1])
        apart = FT._apart(FT._memory(views[0]), FT._memory(views[1]))
        assert apart == (not meet), [(v.dtype, v.shape, v.stride(), v.storage_offset()) for v in views]
        shared += meet and not same
    assert 200 < shared < 2800


def test_no_memory_to_look_at():
    """Tensors of the meta device lie nowhere."""
    assert FT.clip_grad_norm([torch.ones(3, device="meta"), torch.ones(2, device="meta")], 1.0).shape == ()
    assert FT.clip_grad_norm([torch._efficientzerotensor(3), torch.ones(4), torch._efficientzerotensor(4)]) == 2.0
