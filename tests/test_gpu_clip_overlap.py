"""Clipping tensors that share memory on the GPU: the kernels, copies before them and the torch expressions
agree on what counts once and on what is refused."""
import math

import pytest

from gpu_util import dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
FT = pytest.importorskip("paper_2410_15352_amd.finetune")

f16, bf16, f32, f64 = torch.float16, torch.bfloat16, torch.float32, torch.float64


# what else is in the list decides which form answers
BESIDE = {"kernels": lambda: [], "copied": lambda: [torch.zeros(4, 8, device=dev())[:, :5]], "expressions": lambda: [torch.zeros(3, dtype=f64, device=dev())]}


@pytest.mark.parametrize("beside", list(BESIDE))
@pytest.mark.parametrize("dtype", [f16, bf16, f32])
def test_the_same_elements_count_once(beside, dtype):
    for again in (lambda x: x, lambda x: x.view(4, 6), lambda x: x.view(4, 6).t(), lambda x: x.view(2, 3, 4).permute(2, 0, 1)):
        x = torch.full((24,), 2.0, dtype=dtype, device=dev())
        got = FT.clip_grad_norm([x, *BESIDE[beside](), again(x)], 1.0)
        assert math.isclose(float(got), 2 * 24 ** 0.5, rel_tol=1e-6)
        assert ((x.double() - 24 ** -0.5).abs() <= (torch.finfo(dtype).eps / 2 + 2e-7) * 24 ** -0.5).all()


@pytest.mark.parametrize("beside", list(BESIDE))
@pytest.mark.parametrize("bound", [None, 1.0])
def test_a_part_shared_is_refused(beside, bound):
    b = torch.ones(100, device=dev())
    m = b.view(10, 10)
    for pair in ((b[:60], b[40:]), (b, b[10:20]), (m[:, :6], m[:, 4:]), (m[:, 3], m[4]), (b, b.view(bf16))):
        with pytest.raises(ValueError, match="overlap"):
            FT.clip_grad_norm([*BESIDE[beside](), *pair], bound)
    assert (b == 1).all()


@pytest.mark.parametrize("beside", list(BESIDE))
def test_slices_beside_one_another(beside):
    m = torch.ones(64, 96, device=dev())
    t = [m[:32, :40], m[:32, 40:], m[32:, ::2], m[32:, 1::2], m[:0]]
    got = FT.clip_grad_norm([*t, *BESIDE[beside](), t[1].t()], 1.0)
    assert math.isclose(float(got), m.numel() ** 0.5, rel_tol=1e-6) and (m - m.numel() ** -0.5).abs().max() < 1e-8


def test_a_norm_that_is_kept_keeps_nothing_else():
    t = [torch.ones(1 << 22, device=dev()) for _ in range(3)]
    norms = [FT.clip_grad_norm(t, bound) for bound in (None, 1e9, 1.0)]
    assert all(n.untyped_storage().nbytes() <= 16 for n in norms)
