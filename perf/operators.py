"""Performance cases of the expert layers and of their calibration, through the Python binding.

A model with expert layers keeps one delta per expert and sorts its tokens by expert; the same call
serves prompts for several fine-tunes of one base, where the "experts" share the base weights.
Fitting the scales of such layers against a teacher runs the four kinds of work one after another:

  linear   Y[m] = X[m] W_hat_e^T for the tokens m of every expert e
  distill  loss of the student's logits against the teacher's top logits, and its gradient
  grad_x   dX[m] = dY[m] W_hat_e, the gradient that goes on to the layer below
  grad_v   gradient with respect to every expert's scale vector

A case is a plain dict; ``prepare`` builds what a program holds before the call and ``run`` is one
call.  With ``own`` false the call is the plain form: elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
ROW, COL = 0, 1                            # one scale per output feature, or per input feature


def _layer(kind, experts, M, d_out, d_in, dtype, scales, base="own", tail=0):
    return {"kind": kind, "experts": experts, "M": M, "d_out": d_out, "d_in": d_in, "dtype": dtype, "scales": scales,
            "base": base, "tail": tail}


def _loss(T, V, k, dtype, grad, temperature=1.0, masked=False):
    return {"kind": "distill", "T": T, "V": V, "k": k, "dtype": dtype, "grad": grad, "temperature": temperature, "masked": masked}


def listed():
    return [
        # four tokens, two experts each, on the smallest layer of the test configurations: launch and host latency
        {"name": "decode_small", **_layer("linear", 8, 8, 256, 512, "f16", "row")},
        # decode of 32 sequences, two experts of 32 each: every expert that is met is read once
        {"name": "decode_32", **_layer("linear", 32, 64, 2048, 4096, "bf16", "row")},
        # prompts of odd lengths for twelve fine-tunes of one base, in one call
        {"name": "variants_prompt", **_layer("linear", 12, 1501, 4096, 4096, "f16", "col", base="shared")},
        # a prompt of 2048 tokens through eight experts, two for each token: the gate projection
        {"name": "experts_prompt", **_layer("linear", 8, 4096, 14336, 4096, "bf16", "row")},
        # backward through one dense down projection, an odd number of calibration tokens
        {"name": "grad_x_dense", **_layer("grad_x", 1, 777, 4096, 11008, "f16", "row", base="shared")},
        # a small layer whose sizes are no multiple of a tile, and rows of padding behind the last token
        {"name": "grad_x_ragged", **_layer("grad_x", 5, 203, 1001, 1056, "bf16", "row", tail=21)},
        # backward through eight experts' down projections, 2048 tokens, two experts for each
        {"name": "grad_x_experts", **_layer("grad_x", 8, 4096, 4096, 14336, "bf16", "col")},
        # scales of sixteen small experts
        {"name": "grad_v_small", **_layer("grad_v", 16, 515, 2048, 1024, "f16", "row")},
        # scales of eight experts' gate projections
        {"name": "grad_v_experts", **_layer("grad_v", 8, 4096, 14336, 4096, "bf16", "col")},
        # three tokens of a student that answers in 32 bits; an odd vocabulary
        {"name": "distill_small", **_loss(3, 32001, 8, "f32", True)},
        # validation: the loss alone
        {"name": "distill_validate", **_loss(640, 32000, 20, "f16", False, temperature=2.0)},
        # calibration on 2048 tokens of a large vocabulary, the prompt's tokens without weight
        {"name": "distill_train", **_loss(2048, 128256, 64, "bf16", True, masked=True)},
    ]


MAX_FLOPS = 2 * 4096 * 14336 * 4096        # of the largest listed layer
MAX_WEIGHTS = 8 * 14336 * 4096
MAX_LOGITS = 2048 * 128256


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _features(rng, lo, hi, step):
    return max(step, int(round(_log(rng, lo, hi) / step)) * step)


def draw(rng):
    """One more case: layers of 256 to 14336 outputs (any whole number now and then) and 256 to 14336 inputs
    (mostly a multiple of 128, always of 32, the packing's own rule), 1 to 64 experts, 1 to 4096 tokens;
    losses of 1 to 4096 tokens over 1000 to 151936 words."""
    kind = rng.choice(("linear", "linear", "grad_x", "grad_v", "distill", "distill"))
    if kind == "distill":
        dtype = rng.choice(("f16", "bf16", "bf16", "f32"))
        V = int(_log(rng, 1000, 151937))
        if rng.random() < 0.5:
            V = V // 64 * 64
        T = max(1, min(int(_log(rng, 1, 4097)), MAX_LOGITS // V // (2 if dtype == "f32" else 1)))
        return _loss(T, V, int(_log(rng, 1, 129)), dtype, rng.random() < 0.75, rng.choice((1.0, 1.0, 2.0, 0.7)), rng.random() < 0.5)
    dtype = rng.choice(("f16", "bf16"))
    d_out = rng.randint(256, 4096) if rng.random() < 0.25 else _features(rng, 256, 14336, 64)
    d_in = _features(rng, 256, 14336, 32 if rng.random() < 0.25 else 128)
    experts = min(int(_log(rng, 1, 65)), max(1, MAX_WEIGHTS // (d_out * d_in)))
    M = max(1, min(int(_log(rng, 1, 4097)), MAX_FLOPS // (2 * d_out * d_in)))
    base = "shared" if experts == 1 or (kind != "grad_v" and rng.random() < 0.25) else "own"
    tail = 0 if experts == 1 or rng.random() < 0.75 else rng.randint(1, 40)
    return _layer(kind, experts, M, d_out, d_in, dtype, rng.choice(("row", "col")), base, tail)


# ---- inputs -----------------------------------------------------------------------------------

def _counts(case):
    """Tokens of each expert: uneven, now and then none, as a router or a queue of prompts leaves them."""
    rng = random.Random("%(experts)d %(M)d %(d_out)d %(d_in)d" % case)
    load = [0.0 if rng.random() < 0.08 else math.exp(rng.gauss(0.0, 0.45)) for _ in range(case["experts"])]
    if not any(load):
        load[0] = 1.0
    total, given, counts = sum(load), 0, []
    for k in range(case["experts"]):
        upto = case["M"] if k == case["experts"] - 1 else int(round(case["M"] * sum(load[:k + 1]) / total))
        counts.append(upto - given)
        given = upto
    return counts


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g, dtype = _generator(seed), DTYPES[case["dtype"]]

    def normal(shape, scale):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale)

    if case["kind"] == "distill":
        T, V, k = case["T"], case["V"], case["k"]
        logits = normal((T, V), 2.5).to(dtype)
        # a teacher that mostly agrees: its best words by its own logits
        teacher = logits.float().add_(normal((T, V), 0.7))
        top_logits, top_ids = torch.topk(teacher, k, dim=1)
        del teacher
        top_ids = top_ids.to(torch.int32)
        weight = None
        if case["masked"]:
            # the prompt's tokens carry no weight, some rows hold fewer of the teacher's words or none, and the
            # last words of the vocabulary are padding that no row may answer with
            weight = (torch.rand(T, generator=g, device=DEV) < 0.7).float()
            held = torch.randint(0, 2 * k + 1, (T, 1), generator=g, device=DEV)
            top_ids = torch.where(torch.arange(k, device=DEV) < held, top_ids, -1)
            pad = min(17, V - 900)
            logits[:, V - pad:] = float("-inf")
            top_ids = torch.where(top_ids < V - pad, top_ids, -1)
        return {"case": case, "logits": logits, "ids": top_ids, "top": top_logits.to(dtype), "weight": weight,
                "grad_scale": 256.0 if case["dtype"] == "f16" else 1.0}

    E, M, d_out, d_in = case["experts"], case["M"], case["d_out"], case["d_in"]
    counts = _counts(case)
    random.Random(seed).shuffle(counts)
    offsets = [0]
    for n in counts:
        offsets.append(offsets[-1] + n)
    rows = M + case["tail"]
    own_base = () if case["base"] == "shared" else (E,)
    st = {"case": case, "most": max(counts), "offsets": torch.tensor(offsets, dtype=torch.int32).to(DEV)}
    st["B"] = torch.randint(-2 ** 31, 2 ** 31, (E, d_out, d_in // 32), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    # mean |dW| of a delta whose standard deviation is log-normal from channel to channel
    v = normal((E, d_out if case["scales"] == "row" else d_in), 0.5).add_(math.log(1e-3)).exp_().mul_(math.sqrt(2 / math.pi))
    st["v"] = v.to(torch.float16)
    if case["kind"] != "grad_v":
        st["W_b"] = torch.empty(own_base + (d_out, d_in), dtype=dtype, device=DEV)
        st["W_b"].view(-1, d_out * d_in).copy_(normal(own_base + (d_out, d_in), 0.02).view(-1, d_out * d_in))
    if case["kind"] != "grad_x":
        st["X"] = normal((rows, d_in), 1.0).to(dtype)
    if case["kind"] != "linear":
        # gradients of a mean over many tokens are small, and differ in size from token to token
        st["dY"] = (normal((rows, d_out), 1e-3) * normal((rows, 1), 1.0).exp_()).to(dtype)
    if case["kind"] != "grad_v":
        # the program's own activation buffer; rows of padding in it stay as they are
        st["out"] = torch.zeros((rows, d_out if case["kind"] == "linear" else d_in), dtype=dtype, device=DEV)
    return st


# ---- one pass ---------------------------------------------------------------------------------

def _signs(B):
    """+1 and -1 in 32 bits from the packed words [..., d_in / 32]."""
    bits = (B.unsqueeze(-1) >> torch.arange(32, dtype=torch.int32, device=B.device)) & 1
    return bits.flatten(-2).float().mul_(2.0).sub_(1.0)


def _weights(W_b, B, v, scales):
    """W_hat = W_b + v B of every expert, in 32 bits."""
    return _signs(B).mul_(v.float().unsqueeze(2 if scales == "row" else 1)).add_(W_b.float())


def _places(st, rows):
    """Of every row its expert and its place there, and whether it has one."""
    offsets, E = st["offsets"].long(), st["case"]["experts"]
    m = torch.arange(rows, device=offsets.device)
    expert = torch.searchsorted(offsets[1:].contiguous(), m, right=True).clamp_(max=E - 1)
    return expert, (m - offsets[expert]).clamp_(max=st["most"] - 1), (m < offsets[E]).unsqueeze(1)


def _by_expert(st, t):
    """The rows of every expert one behind the other, padded with zeros: [E, most, n]."""
    offsets = st["offsets"].long()
    at = offsets[:-1].unsqueeze(1) + torch.arange(st["most"], device=t.device)
    real = at < offsets[1:].unsqueeze(1)
    return t.float()[at.clamp_(max=t.shape[0] - 1)] * real.unsqueeze(2)


def _plain_distill(st):
    case, tau = st["case"], st["case"]["temperature"]
    z = st["logits"].float() / tau
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    ids = st["ids"].long()
    real = ids >= 0
    ids = ids.clamp(min=0)
    t = torch.where(real, st["top"].float() / tau, float("-inf"))
    best = t.amax(1, keepdim=True)
    best = torch.where(best == float("-inf"), 0.0, best)
    p = (t - best).exp()
    mass = p.sum(1, keepdim=True)
    some = mass > 0
    p = p / torch.where(some, mass, 1.0)
    log_p = t - best - torch.where(some, mass, 1.0).log()
    log_q = z.gather(1, ids) - top - total.log()
    weight = torch.ones_like(top) if st["weight"] is None else st["weight"].unsqueeze(1)
    loss = (torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1, keepdim=True) * (tau * tau) * weight).squeeze(1)
    if not case["grad"]:
        return {"loss": loss}
    grad = (e / total).scatter_add_(1, ids, -p) * (some * weight * (tau * st["grad_scale"]))
    return {"loss": loss, "grad": grad.to(st["logits"].dtype)}


def run(st):
    case = st["case"]
    kind, scales = case["kind"], case.get("scales")
    if own:
        from paper_2512_19720_amd import binding as pd
        if kind == "distill":
            loss, grad = pd.pdelta_distill(st["logits"], st["ids"], st["top"], weight=st["weight"], temperature=case["temperature"],
                                           grad_scale=st["grad_scale"], want_grad=case["grad"])
            return {"loss": loss, "grad": grad} if case["grad"] else {"loss": loss}
        axis = pd.ROW if scales == "row" else pd.COL
        if kind == "linear":
            return pd.pdelta_linear_experts(st["X"], st["offsets"], st["W_b"], st["B"], st["v"], axis, out=st["out"])
        if kind == "grad_x" and case["experts"] == 1:
            return pd.pdelta_grad_x(st["dY"], st["W_b"], st["B"][0], st["v"][0], axis, out=st["out"])
        if kind == "grad_x":
            return pd.pdelta_grad_x_experts(st["dY"], st["offsets"], st["W_b"], st["B"], st["v"], axis, out=st["out"])
        return pd.pdelta_grad_v_experts(st["X"], st["dY"], st["offsets"], st["B"], axis)
    if kind == "distill":
        return _plain_distill(st)
    if kind == "grad_v":
        X, dY, S = _by_expert(st, st["X"]), _by_expert(st, st["dY"]), _signs(st["B"])
        if scales == "row":
            return (dY * torch.bmm(X, S.transpose(1, 2).contiguous())).sum(1)
        return (X * torch.bmm(dY, S)).sum(1)
    W = _weights(st["W_b"], st["B"], st["v"], scales)
    if kind == "linear":
        got = torch.bmm(_by_expert(st, st["X"]), W.transpose(1, 2))
    else:
        got = torch.bmm(_by_expert(st, st["dY"]), W)
    out = st["out"]
    expert, place, real = _places(st, out.shape[0])
    out.copy_(torch.where(real, got[expert, place], out.float()))
    return out


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    """Bytes: logits, tokens, and the weights, sign words and scales of every expert that has tokens once in,
    every result once out."""
    if case["kind"] == "distill":
        T, V, k = case["T"], case["V"], case["k"]
        size = 4 if case["dtype"] == "f32" else 2
        nbytes = T * V * size * (2 if case["grad"] else 1) + T * k * (4 + size) + T * 4 * (2 if case["masked"] else 1)
        return {"bytes": nbytes, "flops": T * V * (6 if case["grad"] else 4)}
    M, d_out, d_in = case["M"], case["d_out"], case["d_in"]
    met = sum(1 for n in _counts(case) if n > 0)
    v_len = d_out if case["scales"] == "row" else d_in
    nbytes = met * (d_out * d_in // 8) + 2 * M * (d_out + d_in) + 4 * (case["experts"] + 1)
    if case["kind"] == "grad_v":
        nbytes += case["experts"] * 4 * v_len
    else:
        nbytes += met * 2 * v_len + (1 if case["base"] == "shared" else met) * 2 * d_out * d_in
    return {"bytes": nbytes, "flops": 2 * M * d_out * d_in}


# ---- the same results in 64 bits ----------------------------------------------------------------

def _signs64(words, d_in):
    """words [d_out, d_in / 32]: input i is bit i % 32 of word i / 32, set for +1."""
    i = torch.arange(d_in, device=words.device)
    return torch.where((words[:, i // 32] >> (i % 32).to(torch.int32)) & 1 == 1, 1.0, -1.0).double()


def _exact_distill(st):
    case, tau = st["case"], st["case"]["temperature"]
    losses, grads = [], []
    for a in range(0, case["T"], 256):
        z = st["logits"][a:a + 256].double() / tau
        log_q = torch.log_softmax(z, 1)
        ids, t = st["ids"][a:a + 256].long(), st["top"][a:a + 256].double() / tau
        t[ids < 0] = float("-inf")
        empty = (ids >= 0).sum(1, keepdim=True) == 0
        p = torch.softmax(t.masked_fill(empty, 0.0), 1).masked_fill(empty | (ids < 0), 0.0)
        target = torch.zeros_like(z).scatter_add_(1, ids.clamp(min=0), p)
        share = torch.xlogy(p, p) - p * torch.where(p > 0, log_q.gather(1, ids.clamp(min=0)), 0.0)
        w = torch.ones(z.shape[0], 1, dtype=torch.float64, device=z.device)
        if st["weight"] is not None:
            w = st["weight"][a:a + 256].double().unsqueeze(1)
        losses.append(tau * tau * w[:, 0] * share.sum(1))
        if case["grad"]:
            grads.append(tau * st["grad_scale"] * w * (log_q.exp() * (~empty) - target))
    loss = torch.cat(losses)
    return {"loss": loss, "grad": torch.cat(grads)} if case["grad"] else {"loss": loss}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "distill":
        return _exact_distill(st)
    E, d_in, offsets = case["experts"], case["d_in"], st["offsets"].tolist()
    row = case["scales"] == "row"
    if case["kind"] == "grad_v":
        out = torch.zeros_like(st["v"], dtype=torch.float64)
    else:
        out = st["out"].double()
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if a == b:
            continue
        W = _signs64(st["B"][e], d_in)
        if case["kind"] == "grad_v":
            dW = st["dY"][a:b].double().T.contiguous() @ st["X"][a:b].double()
            out[e] = (dW * W).sum(1 if row else 0)
            continue
        W *= st["v"][e].double()[:, None] if row else st["v"][e].double()[None, :]
        W += (st["W_b"] if case["base"] == "shared" else st["W_b"][e]).double()
        out[a:b] = st["X"][a:b].double() @ W.T if case["kind"] == "linear" else st["dY"][a:b].double() @ W
    return out
