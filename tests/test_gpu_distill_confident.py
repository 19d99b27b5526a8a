"""GPU: the loss and the gradient of tokens whose student is sure of the teacher's word, where both are close to 0.

With one word far above the others and a teacher that names it alone, loss = log(1 + S) and gradient = -S / (1 + S) at the word, S
the sum of the others' exponentials relative to it.  Relative to the row's true largest logit its own exponential is exactly 1.
What is added to a sum that holds it is a part of S each time, and an addition is off by no more than what is added (1 itself is
a number of the format): the sum is off by at most S, beside the relative error of S itself, 2^-16 at most.  S is chosen to be a few
u = 2^-24.  The logarithm and the quotient of a number this close to 1 are off by at most u each.  Bounds: S + 2 u for the loss and
S + 3 u for the gradient, plus the rounding to the gradient's type."""
import math

import pytest
import torch

from experts_util import U, half_step
from paper_2512_19720_amd import binding as pd
from test_gpu_distill import check, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("T,V", [(40, 8203), (40, 20000), (130, 128256), (9, 128256)])
def test_a_student_that_is_sure(T, V, dtype):
    g = torch.Generator(device=DEV).manual_seed(V + T)
    logits = torch.randn(T, V, generator=g, device=DEV) * 0.3
    at = torch.randint(2 * V // 3, V, (T,), generator=g, device=DEV)
    rows = torch.arange(T, device=DEV)
    logits[rows, at] = math.log(V / (4 * U)) + 0.25 * torch.rand(T, generator=g, device=DEV)
    logits = logits.to(dtype)
    z = logits.double()
    e = (z - z[rows, at, None]).exp()
    e[rows, at] = 0
    S = e.sum(1)
    assert bool((S < 8 * U).all()) and bool((S > U).all())
    scale = 1024.0
    loss, grad = pd.pdelta_distill(logits, at[:, None].to(torch.int32), torch.zeros(T, 1, device=DEV), None, 1.0, scale)
    assert bool(((loss.double() - S.log1p()).abs() <= S + 2 * U).all()), float(((loss.double() - S.log1p()).abs() / (S + 2 * U)).max())
    rel, least = half_step(dtype)
    want = -scale * S / (1 + S)
    bound = scale * (S + 3 * U)
    bound = bound + (want.abs() + bound) * rel + least
    off = (grad[rows, at].double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


@pytest.mark.parametrize("T,V,dtype", [(129, 122880, BF16), (130, 122881, F16), (129, 122889, BF16), (129, 49152, F32), (130, 49157, F32)])
def test_rows_at_the_ends_of_what_is_kept(T, V, dtype):
    """Rows that end where threads begin to keep more of them; some whose largest logits come last."""
    logits, ids, top, g = make(T, V, 5, dtype, T + V)
    logits[1::3, :V - 5] -= 40
    logits[2::5, :V // 2] = float("-inf")
    top[logits.gather(1, ids.long()).isinf()] = float("-inf")
    check(logits, ids, top, None, 0.8, 2.0, f"{T}x{V} {dtype}")
