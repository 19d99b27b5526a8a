"""The operators on tokens sorted by expert and the loss against a teacher's top logits in 64 bits, on the CPU, and bounds
on what the kernels' roundings may add up to.

Bounds, entry by entry (u = 2^-24, one rounding in fp32; h = 2^-11, one rounding to fp16):
  products  Every weight of W_hat is rounded to fp16 once, and a weight below 2^-14 to a multiple of 2^-24; bf16 weights
            are truncated to multiples of 2^-24 as well (fp16 holds their 8 bits elsewhere).  In decode the operand x v
            is rounded to fp16 instead, of the delta term alone.  A token's elements are exact, or off by 2^-38 of the
            row's largest.  A sum of K products in fp32 is off by at most K u of the products' magnitudes.  The result
            is rounded once to its type.
  grad_v    Products are exact; a term takes part in at most D fp32 additions, one per token of the expert, 64 inside a
            tile and its waves, and one per tile of the summed dimension.
  loss      See distill_bounds.
"""
import numpy as np
import torch

U, H = 2.0 ** -24, 2.0 ** -11
ROW, COL = 0, 1


def half_step(dtype):
    """Largest relative error of one rounding, and the largest absolute one next to zero."""
    return {torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float32: (2.0 ** -24, 2.0 ** -150)}[dtype]


def signs64(B, d_in):
    """+1 / -1 from words [..., d_out, d_in / 32]; input i is bit i % 32 of word i / 32."""
    words = B.cpu().numpy().view(np.uint32)
    bits = (words[..., None] >> np.arange(32, dtype=np.uint32)) & 1
    return torch.from_numpy(np.where(bits.reshape(*words.shape[:-1], d_in) == 1, 1.0, -1.0))


def weights64(W_b, B, v, axis, e):
    """W_hat of expert e and the magnitude |W_b| + |v| that its roundings are relative to."""
    S = signs64(B[e], W_b.shape[-1])
    base = (W_b if W_b.dim() == 2 else W_b[e]).cpu().double()
    ve = v[e].cpu().double()
    ve = ve[:, None] if axis == ROW else ve[None, :]
    return base + ve * S, base.abs() + ve.abs()


def spans(offsets):
    o = [int(x) for x in offsets.cpu()]
    return [(e, o[e], o[e + 1]) for e in range(len(o) - 1) if o[e + 1] > o[e]]


def product64(tokens, offsets, W_b, B, v, axis, grad, out_dtype):
    """(values, bound, rows that belong to an expert) of the forward product or of the gradient with respect to the input."""
    t = tokens.cpu().double()
    width = W_b.shape[-1] if grad else W_b.shape[-2]
    ref, bound = torch.zeros(t.shape[0], width, dtype=torch.float64), torch.zeros(t.shape[0], width, dtype=torch.float64)
    mine = torch.zeros(t.shape[0], dtype=torch.bool)
    rel, least = half_step(out_dtype)
    K = t.shape[1]
    for e, a, b in spans(offsets):
        W, size = weights64(W_b, B, v, axis, e)
        if not grad:
            W, size = W.T, size.T
        ref[a:b] = t[a:b] @ W
        mag = t[a:b].abs()
        far = mag.amax(1, keepdim=True) * 2.0 ** -38
        bound[a:b] = (mag @ size) * (H + (K + 8) * U) + mag.sum(1, keepdim=True) * (3 * U) + far * size.sum(0, keepdim=True)
        bound[a:b] = bound[a:b] * (1 + rel) + ref[a:b].abs() * rel + least
        mine[a:b] = True
    return ref, bound, mine


def grad_v64(X, dY, offsets, B, axis):
    X, dY, E, d_in = X.cpu().double(), dY.cpu().double(), B.shape[0], X.shape[1]
    d_out = dY.shape[1]
    kept, summed = (d_out, d_in) if axis == ROW else (d_in, d_out)
    ref, bound = torch.zeros(E, kept, dtype=torch.float64), torch.zeros(E, kept, dtype=torch.float64)
    for e, a, b in spans(offsets):
        D, S = dY[a:b].T @ X[a:b], signs64(B[e], d_in)
        ref[e] = (D * S).sum(1 if axis == ROW else 0)
        size = (dY[a:b].abs().T @ X[a:b].abs()).sum(1 if axis == ROW else 0)
        bound[e] = size * (b - a + 64 + (summed + 63) // 64) * U + 2.0 ** -140
    return ref, bound


def distill64(logits, ids, top, weight, temperature, grad_scale):
    """(loss, grad) in 64 bits, row by row, slot by slot."""
    T, V = logits.shape
    z, t, ids = logits.cpu().double() / temperature, top.cpu().double() / temperature, ids.cpu().tolist()
    w = [1.0] * T if weight is None else weight.cpu().double().tolist()
    loss, grad = torch.zeros(T, dtype=torch.float64), torch.zeros(T, V, dtype=torch.float64)
    for r in range(T):
        slots = [j for j, i in enumerate(ids[r]) if 0 <= i < V and t[r, j] != float("-inf")]
        if w[r] == 0 or not slots:
            continue
        p = torch.softmax(t[r, slots], 0)
        nothing = bool((z[r] == float("-inf")).all())
        log_q = torch.full((V,), float("-inf"), dtype=torch.float64) if nothing else torch.log_softmax(z[r], 0)
        grad[r] = log_q.exp()
        for j, s in enumerate(slots):
            if p[j] > 0:
                loss[r] += p[j] * (p[j].log() - log_q[ids[r][s]])
            grad[r, ids[r][s]] -= p[j]
        loss[r] *= temperature ** 2 * w[r]
        grad[r] *= grad_scale * temperature * w[r]
    return loss, grad


def distill_bounds(logits, ids, top, weight, temperature, grad_scale):
    """An exponential's argument x / tau is formed with three roundings of numbers up to R = (largest - smallest) / tau that
    counts (below -104 an fp32 exponential is 0), and rounded itself; a sum over the vocabulary adds up to V / 64 terms one
    after another; logarithms and the sum over the slots are of numbers up to R + 20, with k more additions."""
    T, V = logits.shape
    finite = logits.cpu().double().masked_fill(~torch.isfinite(logits.cpu()), float("nan"))
    spread = torch.nan_to_num(torch.from_numpy(np.nanmax(finite.numpy(), 1) - np.nanmin(finite.numpy(), 1)), nan=0.0) / temperature
    tt = top.cpu().double().masked_fill(~torch.isfinite(top.cpu()), 0.0)
    R = spread + (tt.amax(1) - tt.amin(1)) / temperature + 20
    w = torch.ones(T, dtype=torch.float64) if weight is None else weight.cpu().double().abs()
    k = top.shape[1]
    delta = U * (6 * torch.clamp(R, max=130) + V / 64 + k + 40)
    loss = w * temperature ** 2 * (delta + 4 * U * R * (1 + k / 16))
    _, grad = distill64(logits, ids, top, None, temperature, grad_scale)
    share = torch.zeros(T, V, dtype=torch.float64)
    for r in range(T):
        for i in ids[r].cpu().tolist():
            if 0 <= i < V:
                share[r, i] = 1.0
    rel, least = half_step(logits.dtype)
    scale = abs(grad_scale) * temperature * w[:, None]
    grad = grad.abs() * w[:, None] * (rel + delta[:, None] * (1 + rel)) + scale * 2 * share * delta[:, None] * (1 + rel) + scale * 2.0 ** -125 + least
    return loss, grad


def held(got, ref, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, what
    assert torch.isfinite(got).all(), what
    off = (got - ref).abs()
    assert bool((off <= bound).all()), f"{what}: an entry is {float((off / bound).nan_to_num(0).max()):.3g} times its bound off"
