"""GPU: products of tokens sorted by expert, forward and backward, and the gradient of every expert's scales, against the
64-bit forms of experts_util with its bounds."""
import pytest
import torch

from experts_util import COL, ROW, grad_v64, held, product64
from paper_2512_19720_amd import binding as pd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def make(counts, d_out, d_in, dtype, axis, seed, shared=False, before=0, behind=0, dy_scale=1e-3):
    g = torch.Generator().manual_seed(seed)
    E, M = len(counts), before + sum(counts) + behind
    offsets = [before]
    for n in counts:
        offsets.append(offsets[-1] + n)
    c = {"offsets": torch.tensor(offsets, dtype=torch.int32),
         "B": torch.randint(-2 ** 31, 2 ** 31, (E, d_out, d_in // 32), generator=g).to(torch.int32),
         "W_b": (torch.randn((d_out, d_in) if shared else (E, d_out, d_in), generator=g) * 0.02).to(dtype),
         "v": (torch.randn(E, d_out if axis == ROW else d_in, generator=g) * 1e-3).to(F16),          # of either sign
         "X": torch.randn(M, d_in, generator=g).to(dtype),
         "dY": (torch.randn(M, d_out, generator=g) * dy_scale * torch.exp(torch.randn(M, 1, generator=g))).to(dtype)}
    return {k: t.to(DEV) for k, t in c.items()}


def linear(c, axis, out_dtype, **kw):
    return pd.pdelta_linear_experts(c["X"], c["offsets"], c["W_b"], c["B"], c["v"], axis, out_dtype=out_dtype, **kw)


def grad_x(c, axis, out_dtype, **kw):
    return pd.pdelta_grad_x_experts(c["dY"], c["offsets"], c["W_b"], c["B"], c["v"], axis, out_dtype=out_dtype, **kw)


def check_products(c, axis, out_dtype, what):
    for grad, name, tokens in ((False, "linear", c["X"]), (True, "grad_x", c["dY"])):
        width = c["W_b"].shape[-1 if grad else -2]
        out = torch.full((tokens.shape[0], width), 7.0, dtype=out_dtype, device=DEV)
        (grad_x if grad else linear)(c, axis, out_dtype, out=out)
        ref, bound, mine = product64(tokens, c["offsets"], c["W_b"], c["B"], c["v"], axis, grad, out_dtype)
        held(out.cpu()[mine], ref[mine], bound[mine], f"{name} {what}")
        assert (out.cpu()[~mine] == 7.0).all(), f"{name} {what}: a row that belongs to nobody was written"


# (tokens of each expert, d_out, d_in): none and one, tiles and their edges, outputs that are no multiple of anything, inputs
# that are one of 32 only, many experts with few tokens
SHAPES = [([1], 32, 32), ([0, 3, 0, 1], 65, 96), ([5, 0, 64, 65], 130, 160), ([63, 1, 17], 257, 128), ([2] * 70, 48, 256),
          ([130, 0, 257], 300, 384), ([0, 0, 0], 40, 64), ([300], 129, 544), ([16, 17, 15, 1, 0, 33], 272, 640), ([40, 3], 1001, 1056)]


@pytest.mark.parametrize("axis", [ROW, COL])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("counts,d_out,d_in", SHAPES)
def test_products_match(counts, d_out, d_in, dtype, axis):
    c = make(counts, d_out, d_in, dtype, axis, 100 + d_out + d_in, before=d_out % 3, behind=d_in // 32 % 4)
    for out_dtype in (dtype, F32):
        check_products(c, axis, out_dtype, f"{counts} {d_out}x{d_in} {dtype} axis {axis} -> {out_dtype}")


@pytest.mark.parametrize("axis", [ROW, COL])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("counts,d_out,d_in", SHAPES)
def test_grad_v_matches(counts, d_out, d_in, dtype, axis):
    c = make(counts, d_out, d_in, dtype, axis, 200 + d_out + d_in, before=2, behind=3)
    c["X"][:2], c["X"][-3:], c["dY"][:2], c["dY"][-3:] = float("nan"), float("inf"), float("nan"), float("nan")    # nobody's rows
    got = pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], axis)
    ref, bound = grad_v64(c["X"].nan_to_num(0, 0, 0), c["dY"].nan_to_num(0, 0, 0), c["offsets"], c["B"], axis)
    held(got, ref, bound, f"grad_v {counts} {d_out}x{d_in} {dtype} axis {axis}")
    again = pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], axis)
    assert torch.equal(got, again)                    # sums in a fixed order


@pytest.mark.parametrize("axis", [ROW, COL])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_shared_base(dtype, axis):
    c = make([70, 0, 9, 33], 192, 256, dtype, axis, 5, shared=True)
    check_products(c, axis, dtype, f"shared base {dtype} axis {axis}")


@pytest.mark.parametrize("axis", [ROW, COL])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,d_out,d_in", [(1, 33, 64), (77, 320, 256), (200, 1001, 352)])
def test_dense_grad_x(M, d_out, d_in, dtype, axis):
    c = make([M], d_out, d_in, dtype, axis, 6, shared=True)
    got = pd.pdelta_grad_x(c["dY"], c["W_b"], c["B"][0], c["v"][0], axis)
    ref, bound, _ = product64(c["dY"], c["offsets"], c["W_b"], c["B"], c["v"], axis, True, dtype)
    held(got, ref, bound, f"dense grad_x {M} {d_out}x{d_in}")
    assert torch.equal(got, grad_x(c, axis, dtype))   # one expert with all tokens


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e-6, 1e6, 1e30])
def test_bf16_gradients_of_any_size(scale):
    """Far below and far above what fp16 holds; rows of zeros among them."""
    c = make([65, 7], 160, 128, BF16, ROW, 8, dy_scale=scale)
    c["dY"][3], c["dY"][70] = 0, 0
    got = grad_x(c, ROW, F32)
    ref, bound, _ = product64(c["dY"], c["offsets"], c["W_b"], c["B"], c["v"], ROW, True, F32)
    held(got, ref, bound, f"gradients of {scale}")
    assert not got[3].any() and not got[70].any()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_what_is_not_a_number_stays_in_its_row(dtype):
    c = make([40, 30], 96, 128, dtype, COL, 9, behind=2)
    clean_y, clean_x = linear(c, COL, dtype), grad_x(c, COL, dtype)
    for t in (c["X"], c["dY"]):
        t[5, 3], t[50, 7], t[70:] = float("nan"), float("inf"), float("nan")
    for got, clean in ((linear(c, COL, dtype), clean_y), (grad_x(c, COL, dtype), clean_x)):
        others = [m for m in range(70) if m not in (5, 50)]
        assert torch.equal(got[others], clean[others])
        assert got[5].isnan().all() and not got[50].isfinite().any()


def test_offsets_out_of_order_stay_in_bounds():
    """No meaning, but no access outside the buffers: the guards around the outputs hold."""
    c = make([40, 30, 20], 96, 128, BF16, ROW, 10)
    for offsets in ([0, 500, 20, 90], [0, 90, 0, 90], [-7, 10, 90, 90], [90, 40, 20, 0], [2 ** 31 - 1, -2 ** 31, 50, 2 ** 31 - 1]):
        c["offsets"] = torch.tensor(offsets, dtype=torch.int32, device=DEV)
        pad = torch.full((90 + 40, 96), 7.0, dtype=BF16, device=DEV)
        linear(c, ROW, BF16, out=pad[20:110])
        assert (pad[:20] == 7.0).all() and (pad[110:] == 7.0).all()
        padx = torch.full((90 + 40, 128), 7.0, dtype=BF16, device=DEV)
        grad_x(c, ROW, BF16, out=padx[20:110])
        assert (padx[:20] == 7.0).all() and (padx[110:] == 7.0).all()
        assert pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], ROW).shape == (3, 96)


def test_no_tokens():
    c = make([0, 0], 64, 96, F16, ROW, 11)
    assert linear(c, ROW, F16).shape == (0, 64) and grad_x(c, ROW, F16).shape == (0, 96)
    out = torch.full((2, 64), 3.0, device=DEV)
    pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], ROW, out=out)
    assert not out.any()


def test_one_expert_is_the_dense_layer():
    """Against the library's own dense calls: the same weights, one expert."""
    c = make([150], 256, 256, F16, ROW, 12, shared=True)
    Y = pd.pdelta_linear_row(c["X"], c["W_b"], c["B"][0], c["v"][0], out_dtype=F32)
    ref, bound, _ = product64(c["X"], c["offsets"], c["W_b"], c["B"], c["v"], ROW, False, F32)
    held(Y, ref, bound, "dense")
    held(linear(c, ROW, F32), ref, bound, "one expert")
    g = pd.pdelta_grad_v(c["X"], c["dY"], c["B"][0], ROW)
    held(g[None], *grad_v64(c["X"], c["dY"], c["offsets"], c["B"], ROW), "dense grad_v")


def test_another_stream():
    c = make([64, 40], 128, 256, BF16, COL, 13)
    want = [linear(c, COL, BF16), grad_x(c, COL, BF16), pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], COL)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [linear(c, COL, BF16), grad_x(c, COL, BF16), pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], COL)]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_captured_call_follows_the_offsets(dtype):
    """One graph of the three calls, replayed with other tokens and other shares of the experts."""
    axis, M, E = ROW, 96, 3
    c = make([50, 0, 46], 130, 256, dtype, axis, 14)
    def calls():
        return linear(c, axis, dtype), grad_x(c, axis, dtype), pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], axis)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held_out = calls()
    for k, offsets in enumerate(([0, 50, 50, 96], [0, 96, 96, 96], [0, 1, 33, 96], [0, 0, 0, 96])):
        fresh = make([50, 0, 46], 130, 256, dtype, axis, 20 + k)
        for name in ("X", "dY"):
            c[name].copy_(fresh[name])
        c["offsets"].copy_(torch.tensor(offsets, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held_out]
        for a, b in zip(got, calls()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


# few tiles and a long contraction: cut into parts, whose sums are added by a second kernel; d_in and d_out of several hundred to thousands
@pytest.mark.parametrize("axis", [ROW, COL])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("counts,d_out,d_in", [([70], 96, 4096), ([3, 0, 100, 41], 300, 1408), ([1], 4100, 64), ([200, 90], 2050, 128), ([33] * 5, 999, 2944)])
def test_long_contractions(counts, d_out, d_in, dtype, axis):
    c = make(counts, d_out, d_in, dtype, axis, 300 + d_out, before=1, behind=2)
    check_products(c, axis, dtype, f"{counts} {d_out}x{d_in} {dtype} axis {axis}")
    check_products(c, axis, F32, f"{counts} {d_out}x{d_in} {dtype} axis {axis} fp32")
    assert torch.equal(grad_x(c, axis, F32)[1:-2], grad_x(c, axis, F32)[1:-2])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("each", [1, 7, 16, 17, 30, 40])
def test_every_number_of_tokens_of_decode(each, dtype):
    """Experts with fewer and with more tokens than a call's average, on rows longer and shorter than one round of the waves."""
    for d_in, axis in ((256, ROW), (1152, COL), (4096, ROW)):
        c = make([0, each // 2, each, 2 * each, 0, each + 5], 56, d_in, dtype, axis, each, behind=1)
        check_products(c, axis, dtype, f"{each} tokens {d_in} {dtype}")


@pytest.mark.parametrize("axis", [ROW, COL])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("counts,d_out,d_in", [([9, 0, 70, 1], 2600, 2080), ([40] * 9, 1300, 1056), ([200, 3], 1032, 4128)])
def test_grad_v_in_runs(counts, d_out, d_in, dtype, axis):
    """Several tiles of the summed dimension for a workgroup, the last of them a short one; experts of one step and of several."""
    c = make(counts, d_out, d_in, dtype, axis, 400 + d_out, before=3, behind=1)
    got = pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], axis)
    held(got, *grad_v64(c["X"], c["dY"], c["offsets"], c["B"], axis), f"grad_v {counts} {d_out}x{d_in} {dtype} axis {axis}")
    assert torch.equal(got, pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], axis))


@pytest.mark.parametrize("dtype,d_in", [(F16, 96), (BF16, 384)])
def test_many_experts(dtype, d_in):
    """More experts than lanes of a wave, on the decode tiles and on the large ones."""
    counts = [(7 * k) % 41 + 17 for k in range(150)]
    c = make(counts, 72, d_in, dtype, ROW, 17, before=3, behind=5)
    check_products(c, ROW, dtype, f"150 experts {dtype}")
    c = make([k % 3 for k in range(300)], 40, 128, dtype, COL, 18)
    check_products(c, COL, dtype, f"300 experts {dtype}")
    got = pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], COL)
    held(got, *grad_v64(c["X"], c["dY"], c["offsets"], c["B"], COL), "grad_v of 300 experts")


def test_offsets_that_all_name_everything():
    """Many experts that each claim all tokens: sums over them pass 31 bits; no meaning, no access outside the buffers."""
    E, M, d = 2048, 4096, 64
    X = torch.zeros(M, d, dtype=F16, device=DEV)
    offsets = torch.tensor([0, M] * (E // 2) + [0], dtype=torch.int32, device=DEV)
    W = torch.zeros(d, d, dtype=F16, device=DEV)
    B, v = torch.zeros(E, d, d // 32, dtype=torch.int32, device=DEV), torch.zeros(E, d, dtype=F16, device=DEV)
    pad = torch.full((M + 600, d), 7.0, dtype=F16, device=DEV)
    pd.pdelta_linear_experts(X, offsets, W, B, v, ROW, out=pad[300:M + 300])
    assert (pad[:300] == 7.0).all() and (pad[M + 300:] == 7.0).all()
    pd.pdelta_grad_x_experts(X, offsets, W, B, v, ROW, out=pad[300:M + 300])
    assert (pad[:300] == 7.0).all() and (pad[M + 300:] == 7.0).all()


def test_experts_beyond_two_to_the_31_weights():
    """The last expert's weights, signs and tokens like those of a call of their own."""
    E, d_out, d_in = 40, 8192, 8192                   # 2.7e9 weights
    g = torch.Generator(device=DEV).manual_seed(5)
    W = torch.zeros(E, d_out, d_in, dtype=BF16, device=DEV)
    B = torch.zeros(E, d_out, d_in // 32, dtype=torch.int32, device=DEV)
    v = torch.full((E, d_out), 0.001, dtype=F16, device=DEV)
    W[-1] = torch.randn(d_out, d_in, generator=g, device=DEV) * 0.02
    B[-1] = torch.randint(-2 ** 31, 2 ** 31, (d_out, d_in // 32), generator=g, device=DEV).to(torch.int32)
    X = torch.randn(70, d_in, generator=g, device=DEV).to(BF16)
    dY = torch.randn(70, d_out, generator=g, device=DEV).to(BF16)
    for n in (5, 70):                                 # decode tiles and large ones
        offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
        offsets[-1] = n
        one = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        last = (W[-1:].contiguous(), B[-1:].contiguous(), v[-1:].contiguous())
        for grad, t in ((False, X), (True, dY)):
            f = pd.pdelta_grad_x_experts if grad else pd.pdelta_linear_experts
            got, want = f(t[:n], offsets, W, B, v, ROW, out_dtype=F32), f(t[:n], one, *last, ROW, out_dtype=F32)
            # (a call of 40 experts may take other tiles than one of one: each within its bound of the exact value, 2^-11 of the sum of sizes)
            bound = t[:n].abs().float() @ (last[0][0].abs().float() + 0.001).T if not grad else t[:n].abs().float() @ (last[0][0].abs().float() + 0.001)
            assert ((got - want).abs() <= bound * 2.0 ** -10).all()
        gv = pd.pdelta_grad_v_experts(X[:n], dY[:n], offsets, B, ROW)
        assert torch.equal(gv[:-1], torch.zeros_like(gv[:-1]))
        want = pd.pdelta_grad_v_experts(X[:n], dY[:n], one, last[1], ROW)
        assert ((gv[-1] - want[0]).abs() <= want.abs().max() * 1e-4).all()


# tokens around the ends of tiles of 128, 192 and 256; one expert (chosen before the launch) and several (chosen in it); the last three: 192, of one expert in one round
# of tiles on 256 CUs, in two, and of several
@pytest.mark.parametrize("counts,d_out,d_in", [([129], 300, 288), ([192], 520, 256), ([193], 96, 352), ([777], 512, 128), ([385, 0, 191], 260, 512),
                                               ([129, 257, 1], 1024, 288), ([255, 128, 640, 0, 193], 320, 256), ([513, 96], 2050, 96),
                                               ([900], 11008, 160), ([1500], 14336, 160), ([700, 300], 8300, 160)])
def test_tiles_of_every_height(counts, d_out, d_in):
    for k, (dtype, axis) in enumerate([(F16, ROW), (F16, COL), (BF16, ROW), (BF16, COL)]):
        c = make(counts, d_out, d_in, dtype, axis, 900 + k + d_out, before=1, behind=2)
        check_products(c, axis, dtype, f"{counts} {d_out}x{d_in} {dtype} axis {axis}")
    d_out = (d_out + 31) // 32 * 32                     # (inputs come in words of 32)
    c = make(counts, d_in, d_out, F16, ROW, 950 + d_out, before=3)
    check_products(c, ROW, F16, f"{counts} {d_in}x{d_out}")


def test_few_offsets_that_name_the_same_tokens():
    M, d = 700, 128
    X = torch.zeros(M, d, dtype=F16, device=DEV)
    W = torch.zeros(d, d, dtype=F16, device=DEV)
    B, v = torch.zeros(5, d, d // 32, dtype=torch.int32, device=DEV), torch.zeros(5, d, dtype=F16, device=DEV)
    for offsets in ([0, M, 0, M, 0, M], [M, 0, 300, 100, 2 ** 31 - 1, -5]):
        pad = torch.full((M + 600, d), 7.0, dtype=F16, device=DEV)
        o = torch.tensor(offsets, dtype=torch.int32, device=DEV)
        pd.pdelta_linear_experts(X, o, W, B, v, ROW, out=pad[300:M + 300])
        pd.pdelta_grad_x_experts(X, o, W, B, v, ROW, out=pad[300:M + 300])
        assert (pad[:300] == 7.0).all() and (pad[M + 300:] == 7.0).all()


@pytest.mark.parametrize("dtype,out_dtype", [(F16, BF16), (BF16, F16)])
@pytest.mark.parametrize("counts", [[3, 0, 9], [100, 0, 290]])
def test_outputs_of_the_other_type(counts, dtype, out_dtype):
    for axis in (ROW, COL):
        check_products(make(counts, 136, 256, dtype, axis, 31, dy_scale=1.0), axis, out_dtype, f"{counts} {dtype} -> {out_dtype} axis {axis}")


def test_tokens_beyond_two_to_the_31_values():
    """The last expert's tokens, at the end of more than 2^31 values, like those of a call of their own."""
    M, wide, narrow, n = 530000, 4096, 96, 300
    g = torch.Generator(device=DEV).manual_seed(6)
    tokens = torch.zeros(M, wide, dtype=BF16, device=DEV)
    tokens[-n:] = torch.randn(n, wide, generator=g, device=DEV)
    small = torch.zeros(M, narrow, dtype=BF16, device=DEV)
    small[-n:] = torch.randn(n, narrow, generator=g, device=DEV)
    W = (torch.randn(3, narrow, wide, generator=g, device=DEV) * 0.02).to(BF16)
    B = torch.randint(-2 ** 31, 2 ** 31, (3, narrow, wide // 32), generator=g, device=DEV).to(torch.int32)
    v = torch.full((3, narrow), 0.001, dtype=F16, device=DEV)
    offsets = torch.tensor([0, 5, M - n, M], dtype=torch.int32, device=DEV)
    one = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    last = (W[-1:].contiguous(), B[-1:].contiguous(), v[-1:].contiguous())
    # each within a rounding of W_hat and of the fp32 sums of the exact value: 2^-11 of the sum of sizes, and a little
    sizes = W[-1].abs().float() + 0.001
    got, want = pd.pdelta_linear_experts(tokens, offsets, W, B, v, ROW, out_dtype=F32)[-n:], pd.pdelta_linear_experts(tokens[-n:], one, *last, ROW, out_dtype=F32)
    assert ((got - want).abs() <= tokens[-n:].abs().float() @ sizes.T * 2.0 ** -10).all() and want.abs().max() > 0
    gv, alone = pd.pdelta_grad_v_experts(tokens, small, offsets, B, ROW), pd.pdelta_grad_v_experts(tokens[-n:], small[-n:], one, last[1], ROW)
    # sums in fp32 of n products and of `wide` of those
    bound = (small[-n:].abs().float().T @ tokens[-n:].abs().float()).sum(1) * (n + wide) * 2.0 ** -23
    assert torch.equal(gv[:2], torch.zeros_like(gv[:2])) and ((gv[2] - alone[0]).abs() <= bound).all() and alone.abs().max() > 0
    del got, want
    got, want = pd.pdelta_grad_x_experts(small, offsets, W, B, v, ROW)[-n:], pd.pdelta_grad_x_experts(small[-n:], one, *last, ROW)
    bound = small[-n:].abs().float() @ sizes * 2.0 ** -10
    assert ((got.float() - want.float()).abs() <= bound + want.float().abs() * 2.0 ** -7).all() and want.abs().max() > 0     # and two roundings to bf16
