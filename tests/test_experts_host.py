"""Refusals of the entry points for tokens sorted by expert and for the distillation loss, without a GPU."""
import pytest
import torch

from paper_2512_19720_amd import binding as pd

GB = 1 << 30
TOK, OFF, W, B, V, OUT, WS = (k * 8 * GB for k in range(1, 8))       # fake device addresses, never dereferenced
BIG = 4 * GB


def product(fn, tok=TOK, off=OFF, w=W, shared=0, b=B, v=V, axis=pd.ROW, out=OUT, M=100, E=4, d_out=96, d_in=128, dt=pd.F16, odt=pd.F16,
            ws=WS, ws_bytes=BIG):
    return getattr(pd.lib(), fn)(tok, off, w, shared, b, v, axis, out, M, E, d_out, d_in, dt, odt, ws, ws_bytes, None)


@pytest.mark.parametrize("fn", ["pdelta_linear_experts", "pdelta_grad_x_experts"])
def test_product_refusals(fn):
    for null in ("tok", "off", "w", "b", "v", "out"):
        assert product(fn, **{null: None}) == pd.EINVAL, null
    for k, at in dict(tok=TOK, off=OFF, w=W, b=B, v=V, out=OUT, ws=WS).items():
        assert product(fn, **{k: at + 8}) == pd.EALIGN, k
    for bad in (dict(axis=2), dict(axis=-1), dict(M=-1), dict(E=0), dict(E=-3), dict(d_out=0), dict(d_in=0), dict(d_in=-32), dict(shared=2)):
        assert product(fn, **bad) == pd.EINVAL, bad
    for bad in (dict(d_in=100), dict(d_out=(1 << 22) + 1), dict(M=(1 << 23) + 1), dict(E=(1 << 16) + 1)):
        assert product(fn, **bad) == pd.ESHAPE, bad
    assert product(fn, dt=pd.F32) == pd.EDTYPE and product(fn, odt=5) == pd.EDTYPE
    for k, at in dict(tok=TOK, off=OFF, w=W, b=B, v=V).items():
        assert product(fn, out=at) == pd.EINVAL, k                     # the output on an input
        assert product(fn, ws=at) == pd.EINVAL, k                      # the workspace on an input
    assert product(fn, ws=OUT) == pd.EINVAL
    assert product(fn, out=W + 3 * 96 * 128 * 2) == pd.EINVAL          # inside the last expert's weights
    assert product(fn, out=B + 96 * 128 // 8 * 4 - 16) == pd.EINVAL    # the last words of the last expert
    # no tokens: nothing to do, and no tensors needed
    assert product(fn, M=0) == pd.OK and product(fn, M=0, tok=None, out=None, ws=None, ws_bytes=0) == pd.OK


@pytest.mark.parametrize("fn,sizes", [("pdelta_linear_experts", (1000, 4, 96, 128, pd.BF16)), ("pdelta_grad_x_experts", (100, 4, 96, 128, pd.BF16)),
                                      ("pdelta_grad_x_experts", (100, 4, 97, 128, pd.F16))])
def test_product_workspace(fn, sizes):
    M, E, d_out, d_in, dt = sizes
    need = getattr(pd.lib(), fn + "_workspace_bytes")(*sizes)
    assert need > 0
    args = dict(M=M, E=E, d_out=d_out, d_in=d_in, dt=dt)
    assert product(fn, ws_bytes=need - 1, **args) == pd.EWORKSPACE
    assert product(fn, ws=None, ws_bytes=0, **args) == pd.EWORKSPACE
    assert product(fn, ws=None, ws_bytes=need, **args) == pd.EINVAL
    assert getattr(pd.lib(), fn + "_workspace_bytes")(0, *sizes[1:]) == 0
    for bad in ((-1, 4, 96, 128, dt), (100, 0, 96, 128, dt), (100, 4, 0, 128, dt), (100, 4, 96, 100, dt), (100, 4, 96, 128, pd.F32)):
        assert getattr(pd.lib(), fn + "_workspace_bytes")(*bad) == 0


def test_dense_grad_x_refusals():
    def call(tok=TOK, w=W, b=B, v=V, axis=pd.COL, out=OUT, M=100, d_out=96, d_in=128, dt=pd.BF16, odt=pd.F32, ws=WS, n=BIG):
        return pd.lib().pdelta_grad_x(tok, w, b, v, axis, out, M, d_out, d_in, dt, odt, ws, n, None)
    for null in ("tok", "w", "b", "v", "out"):
        assert call(**{null: None}) == pd.EINVAL
    assert call(w=W + 2) == pd.EALIGN and call(d_in=48) == pd.ESHAPE and call(dt=pd.F32) == pd.EDTYPE and call(out=TOK) == pd.EINVAL
    need = pd.lib().pdelta_grad_x_workspace_bytes(100, 96, 128, pd.BF16)
    assert need == pd.lib().pdelta_grad_x_experts_workspace_bytes(100, 1, 96, 128, pd.BF16) > 0
    assert call(n=need - 1) == pd.EWORKSPACE and call(M=0, tok=None, out=None, ws=None, n=0) == pd.OK


def test_grad_v_refusals():
    def call(x=TOK, dy=W, off=OFF, b=B, axis=pd.ROW, out=OUT, M=100, E=4, d_out=97, d_in=128, dt=pd.BF16, ws=WS, n=BIG):
        return pd.lib().pdelta_grad_v_experts(x, dy, off, b, axis, out, M, E, d_out, d_in, dt, ws, n, None)
    for null in ("x", "dy", "off", "b", "out"):
        assert call(**{null: None}) == pd.EINVAL, null
    for k, at in dict(x=TOK, dy=W, off=OFF, b=B, out=OUT, ws=WS).items():
        assert call(**{k: at + 4}) == pd.EALIGN, k
    for bad in (dict(axis=2), dict(M=-1), dict(E=0), dict(d_out=0)):
        assert call(**bad) == pd.EINVAL, bad
    assert call(d_in=33) == pd.ESHAPE and call(E=70000) == pd.ESHAPE and call(dt=pd.F32) == pd.EDTYPE
    for at in (TOK, W, OFF, B):
        assert call(out=at) == pd.EINVAL and call(ws=at) == pd.EINVAL
    assert call(ws=OUT) == pd.EINVAL
    for axis in (pd.ROW, pd.COL):
        need = pd.lib().pdelta_grad_v_experts_workspace_bytes(100, 4, 97, 128, axis)
        assert need > 0 and call(axis=axis, n=need - 1) == pd.EWORKSPACE and call(axis=axis, ws=None, n=0) == pd.EWORKSPACE
    assert pd.lib().pdelta_grad_v_experts_workspace_bytes(100, 4, 97, 128, 2) == 0


def test_distill_refusals():
    def call(z=TOK, ids=OFF, top=W, w=B, loss=V, grad=OUT, T=10, vocab=1000, k=8, dt=pd.BF16, tdt=pd.F32, tau=1.0, scale=1.0, ws=WS, n=BIG):
        return pd.lib().pdelta_distill(z, ids, top, w, loss, grad, T, vocab, k, dt, tdt, tau, scale, ws, n, None)
    for null in ("z", "ids", "top", "loss"):
        assert call(**{null: None}) == pd.EINVAL, null
    for key, at in dict(z=TOK, ids=OFF, top=W, w=B, loss=V, grad=OUT, ws=WS).items():
        assert call(**{key: at + 4}) == pd.EALIGN, key
    nan, inf = float("nan"), float("inf")
    for bad in (dict(T=-1), dict(vocab=0), dict(k=0), dict(tau=0.0), dict(tau=-1.0), dict(tau=nan), dict(tau=inf), dict(scale=nan), dict(scale=inf)):
        assert call(**bad) == pd.EINVAL, bad
    for bad in (dict(k=1025), dict(vocab=(1 << 22) + 1), dict(T=(1 << 23) + 1)):
        assert call(**bad) == pd.ESHAPE, bad
    assert call(dt=3) == pd.EDTYPE and call(tdt=-1) == pd.EDTYPE
    assert call(grad=TOK + 16) == pd.EINVAL                            # on the logits, but not in their place
    for at in (TOK, OFF, W, B, OUT):
        assert call(loss=at) == pd.EINVAL
    for at in (OFF, W, B, V):
        assert call(grad=at) == pd.EINVAL
    assert call(T=0, z=None, ids=None, top=None, w=None, loss=None, grad=None) == pd.OK
    for bad in ((-1, 10, 1, pd.F16), (1, 0, 1, pd.F16), (1, 10, 0, pd.F16), (1, 10, 2000, pd.F16), (1, 10, 1, 9)):
        assert pd.lib().pdelta_distill_workspace_bytes(*bad) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    E, M, d_out, d_in = 3, 8, 40, 64
    ok = dict(X=torch.zeros(M, d_in, dtype=torch.float16), offsets=torch.zeros(E + 1, dtype=torch.int32),
              W_b=torch.zeros(E, d_out, d_in, dtype=torch.float16), B_packed=torch.zeros(E, d_out, 2, dtype=torch.int32),
              v=torch.zeros(E, d_out, dtype=torch.float16), axis=pd.ROW)
    f16, i32 = torch.float16, torch.int32
    bad = [dict(offsets=torch.zeros(E, dtype=i32)), dict(offsets=torch.zeros(E + 1, dtype=torch.int64)), dict(offsets=torch.zeros(1, E + 1, dtype=i32)),
           dict(X=torch.zeros(M, d_in + 32, dtype=f16)), dict(X=torch.zeros(M, d_in)), dict(X=torch.zeros(1, M, d_in, dtype=f16)),
           dict(W_b=torch.zeros(E + 1, d_out, d_in, dtype=f16)), dict(W_b=torch.zeros(E, d_out, d_in, dtype=torch.bfloat16)),
           dict(W_b=torch.zeros(d_in, dtype=f16)), dict(B_packed=torch.zeros(E, d_out, 1, dtype=i32)), dict(B_packed=torch.zeros(E, d_out, 2)),
           dict(B_packed=torch.zeros(d_out, 2, dtype=i32)), dict(v=torch.zeros(E, d_in, dtype=f16)), dict(v=torch.zeros(E, d_out)),
           dict(v=torch.zeros(d_out, dtype=f16)), dict(axis=2), dict(out=torch.zeros(M, d_in, dtype=f16)),
           dict(out=torch.zeros(M, d_out, dtype=f16), out_dtype=torch.float32)]
    for change in bad:
        with pytest.raises(ValueError):
            pd.pdelta_linear_experts(**{**ok, **change})
    with pytest.raises(ValueError):
        pd.pdelta_linear_experts(**ok)                                 # not on a GPU
    with pytest.raises(ValueError):
        pd.pdelta_grad_x(torch.zeros(M, d_out, dtype=f16), ok["W_b"], ok["B_packed"], ok["v"], pd.ROW)         # of several experts
    with pytest.raises(ValueError):
        pd.pdelta_grad_x(torch.zeros(M, d_in, dtype=f16), ok["W_b"][0], ok["B_packed"][0], ok["v"][0], pd.ROW)   # as wide as X
    dY = torch.zeros(M, d_out, dtype=f16)
    for change in (dict(dY=dY[:-1]), dict(dY=dY.float()), dict(axis=3), dict(B_packed=ok["B_packed"][:, :-1]), dict(offsets=ok["offsets"][1:]),
                   dict(out=torch.zeros(E, d_in)), dict(out=torch.zeros(E, d_out, dtype=f16))):
        with pytest.raises(ValueError):
            pd.pdelta_grad_v_experts(**{**dict(X=ok["X"], dY=dY, offsets=ok["offsets"], B_packed=ok["B_packed"], axis=pd.ROW), **change})


def test_binding_refuses_a_loss_that_does_not_fit():
    T, V, k = 5, 30, 4
    ok = dict(logits=torch.zeros(T, V), top_ids=torch.zeros(T, k, dtype=torch.int32), top_logits=torch.zeros(T, k))
    for change in (dict(logits=torch.zeros(1, T, V)), dict(top_ids=torch.zeros(T, k, dtype=torch.int64)), dict(top_ids=torch.zeros(T - 1, k, dtype=torch.int32)),
                   dict(top_logits=torch.zeros(T, k + 1)), dict(weight=torch.zeros(T, 1)), dict(weight=torch.zeros(T, dtype=torch.float16)),
                   dict(out=torch.zeros(T, V), want_grad=False), dict(out=torch.zeros(T, V + 1)), dict(out=torch.zeros(T, V, dtype=torch.float16))):
        with pytest.raises(ValueError):
            pd.pdelta_distill(**{**ok, **change})
    with pytest.raises(ValueError):
        pd.pdelta_distill(**ok)                                        # not on a GPU
