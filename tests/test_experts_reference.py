"""The 64-bit forms that the GPU tests compare with: gradients against central differences of the forward forms."""
import pytest
import torch

from experts_util import COL, ROW, distill64, grad_v64, product64

E, D_OUT, D_IN, OFFSETS = 3, 7, 64, [1, 4, 4, 6]


def make(seed):
    g = torch.Generator().manual_seed(seed)
    B = torch.randint(-2 ** 31, 2 ** 31, (E, D_OUT, D_IN // 32), generator=g).to(torch.int32)
    W_b = torch.randn(E, D_OUT, D_IN, generator=g, dtype=torch.float64)
    X, dY = torch.randn(8, D_IN, generator=g, dtype=torch.float64), torch.randn(8, D_OUT, generator=g, dtype=torch.float64)
    return B, W_b, X, dY, torch.tensor(OFFSETS, dtype=torch.int32), g


def forward(X, offsets, W_b, B, v, axis):
    return product64(X, offsets, W_b, B, v, axis, False, torch.float32)[0]


@pytest.mark.parametrize("axis", [ROW, COL])
def test_gradients_of_the_product_against_differences(axis):
    B, W_b, X, dY, offsets, g = make(axis)
    v = torch.randn(E, D_OUT if axis == ROW else D_IN, generator=g, dtype=torch.float64)
    step = 2.0 ** -10                                 # the product is linear in X and in v: no error of its own beside rounding
    dX = product64(dY, offsets, W_b, B, v, axis, True, torch.float32)[0]
    dv = grad_v64(X, dY, offsets, B, axis)[0]
    for m in range(8):
        for i in (0, 5, 31, 32, 63):
            up, down = X.clone(), X.clone()
            up[m, i] += step
            down[m, i] -= step
            diff = ((forward(up, offsets, W_b, B, v, axis) - forward(down, offsets, W_b, B, v, axis)) * dY).sum() / (2 * step)
            assert abs(float(diff - dX[m, i])) < 1e-9
    for e in range(E):
        for j in range(0, v.shape[1], 3):
            up, down = v.clone(), v.clone()
            up[e, j] += step
            down[e, j] -= step
            diff = ((forward(X, offsets, W_b, B, up, axis) - forward(X, offsets, W_b, B, down, axis)) * dY).sum() / (2 * step)
            assert abs(float(diff - dv[e, j])) < 1e-9
    assert not dX[0].any() and not dX[6:].any() and not dv[1].any()


@pytest.mark.parametrize("temperature", [1.0, 0.7, 3.0])
def test_gradient_of_the_loss_against_differences(temperature):
    g = torch.Generator().manual_seed(7)
    logits = torch.randn(4, 11, generator=g, dtype=torch.float64) * 2
    ids = torch.tensor([[3, 3, 10], [0, -1, 4], [-1, -1, -1], [9, 11, 2]], dtype=torch.int32)
    top = torch.randn(4, 3, generator=g, dtype=torch.float64)
    weight = torch.tensor([1.0, 0.5, 1.0, 2.0])
    loss, grad = distill64(logits, ids, top, weight, temperature, 8.0)
    assert float(loss[2]) == 0 and not grad[2].any()
    step = 2.0 ** -12
    for r in range(4):
        for i in range(11):
            up, down = logits.clone(), logits.clone()
            up[r, i] += step
            down[r, i] -= step
            diff = 8.0 * (distill64(up, ids, top, weight, temperature, 1.0)[0] - distill64(down, ids, top, weight, temperature, 1.0)[0]).sum() / (2 * step)
            assert abs(float(diff - grad[r, i])) < 1e-5


def test_a_student_that_agrees_with_its_teacher_loses_nothing():
    """All words in the slots, the teacher's logits the student's: KL is 0, and so is its gradient."""
    g = torch.Generator().manual_seed(3)
    logits = torch.randn(2, 6, generator=g, dtype=torch.float64)
    ids = torch.stack([torch.randperm(6, generator=g) for _ in range(2)])
    loss, grad = distill64(logits, ids.to(torch.int32), logits.gather(1, ids), None, 2.0, 1.0)
    assert loss.abs().max() < 1e-14 and grad.abs().max() < 1e-14
