"""GPU: one step of fitting the scales of a small model with experts against a teacher's top logits, all calls one after
another as a program makes them, against the same step in 64 bits.

Tolerance: on the way from the logits to the gradients values are rounded to 16 bits four times (hidden states, logits, their
gradient, the hidden states' gradient) and the weights of two layers to fp16 once, each at most 2^-11 of a value in fp16.  A
logit of magnitude up to 8 is off by at most 8 (2 2^-11 + K u) < 0.01, so a share q by 1 %; everything after the loss is linear.
Together below 2 % of a gradient's norm."""
import pytest
import torch

from experts_util import COL, ROW, distill64, signs64
from paper_2512_19720_amd import binding as pd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def packed(g, *shape):
    return torch.randint(-2 ** 31, 2 ** 31, shape, generator=g).to(torch.int32)


@pytest.mark.parametrize("axis", [ROW, COL])
def test_one_step(axis):
    g = torch.Generator().manual_seed(40 + axis)
    T, E, d, hidden, V, k, tau, scale = 90, 5, 256, 320, 1001, 12, 1.5, 512.0
    f16 = torch.float16
    tokens = torch.randn(T, d, generator=g).to(f16)
    router = torch.randint(0, E, (T,), generator=g)
    router[router == 3] = 1                           # nobody goes to expert 3
    W1, B1 = (torch.randn(E, hidden, d, generator=g) * 0.06).to(f16), packed(g, E, hidden, d // 32)
    v1 = (torch.rand(E, hidden if axis == ROW else d, generator=g) * 0.01).to(f16)
    W2, B2 = (torch.randn(V, hidden, generator=g) * 0.1).to(f16), packed(g, V, hidden // 32)
    v2 = (torch.rand(V, generator=g) * 0.01).to(f16)
    top = torch.randn(T, k, generator=g) * 2
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(T)]).to(torch.int32)
    weight = (torch.rand(T, generator=g) < 0.8).float()

    # the program: sort the tokens by expert, forward, loss, backward
    D = {n: t.to(DEV) for n, t in dict(tokens=tokens, router=router, W1=W1, B1=B1, v1=v1, W2=W2, B2=B2, v2=v2, top=top, ids=ids, weight=weight).items()}
    order = torch.argsort(D["router"], stable=True)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = torch.cumsum(torch.bincount(D["router"], minlength=E), 0)
    X = D["tokens"][order]
    H = pd.pdelta_linear_experts(X, offsets, D["W1"], D["B1"], D["v1"], axis)
    logits = pd.pdelta_linear_row(H, D["W2"], D["B2"], D["v2"])
    loss, dlogits = pd.pdelta_distill(logits, D["ids"][order], D["top"][order], D["weight"][order], tau, scale, out=logits)
    dH = pd.pdelta_grad_x(dlogits, D["W2"], D["B2"], D["v2"], ROW)
    dv1 = pd.pdelta_grad_v_experts(X, dH, offsets, D["B1"], axis)
    dX = pd.pdelta_grad_x_experts(dH, offsets, D["W1"], D["B1"], D["v1"], axis)

    # the same in 64 bits, gradients by the chain rule on dense weights
    o = order.cpu()
    x, e = tokens.double()[o], router[o]
    S1, S2 = signs64(B1, d), signs64(B2, hidden)
    scales = v1.double()[:, :, None] if axis == ROW else v1.double()[:, None, :]
    What1, What2 = W1.double() + scales * S1, W2.double() + v2.double()[:, None] * S2
    h = torch.stack([What1[e[m]] @ x[m] for m in range(T)])
    want_loss, dz = distill64(h @ What2.T, ids[o], top[o], weight[o], tau, scale)
    dh = dz @ What2
    dx = torch.stack([dh[m] @ What1[e[m]] for m in range(T)])
    dW = torch.zeros_like(What1)
    for m in range(T):
        dW[e[m]] += dh[m][:, None] * x[m][None, :]
    dv = (dW * S1).sum(2 if axis == ROW else 1)
    assert (loss.cpu().double() - want_loss).abs().max() < 0.02 * want_loss.abs().max()
    for got, ref, what in ((dX, dx, "dX"), (dv1, dv, "dv")):
        assert float((got.cpu().double() - ref).norm() / ref.norm()) < 0.02, what
    assert not dv1[3].any()

    # and dv against differences of the loss in 64 bits, along the gradient itself
    direction, step = dv / dv.norm(), 1e-4
    def total(v):
        s = v[:, :, None] if axis == ROW else v[:, None, :]
        W = W1.double() + s * S1
        z = torch.stack([W[e[m]] @ x[m] for m in range(T)]) @ What2.T
        return float(distill64(z, ids[o], top[o], weight[o], tau, 1.0)[0].sum())
    diff = scale * (total(v1.double() + step * direction) - total(v1.double() - step * direction)) / (2 * step)
    assert abs(diff / float((dv1.cpu().double() * direction).sum()) - 1) < 0.03
