"""GPU: the calls on tokens sorted by expert and the loss in a workspace of exactly the bytes that the library asks for, whatever it
holds, with its surroundings left alone; tokens that are not a number on the decode tiles."""
import pytest
import torch

from experts_util import COL, ROW
from paper_2512_19720_amd import binding as pd
from test_gpu_distill import make as make_loss
from test_gpu_experts import make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
EDGE = 4096


def in_exactly(need, call, want):
    """`call` in a workspace of `need` bytes of NaN patterns."""
    assert need > 0
    memory = torch.full((EDGE + need + EDGE,), 0xFF, dtype=torch.uint8, device=DEV)
    for fill in (0xFF, 0x7F, 0x00):
        memory[EDGE:EDGE + need] = fill
        got = call(memory[EDGE:EDGE + need])
        for a, b in zip(got, want):
            assert torch.equal(a, b), fill
        assert bool((memory[:EDGE] == 0xFF).all()) and bool((memory[EDGE + need:] == 0xFF).all()), fill
    with pytest.raises(pd.PdeltaError):
        call(memory[EDGE:EDGE + need - 1])


# prepared rows, their factors, signs in wider rows and the parts' sums, in all combinations; numbers of tokens that are odd
@pytest.mark.parametrize("axis", [ROW, COL])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("counts,d_out,d_in", [([71], 97, 4128), ([3, 0, 101, 41], 301, 1440), ([333, 18], 1003, 160), ([90] * 7, 2050, 256), ([35, 1], 131, 2080)])
def test_products(counts, d_out, d_in, dtype, axis):
    c = make(counts, d_out, d_in, dtype, axis, 500 + d_out, before=1, behind=2)
    M, E = c["X"].shape[0], len(counts)
    for grad, tokens, width in ((False, c["X"], d_out), (True, c["dY"], d_in)):
        fn = pd.pdelta_grad_x_experts if grad else pd.pdelta_linear_experts
        size = pd.pdelta_grad_x_experts_workspace_bytes if grad else pd.pdelta_linear_experts_workspace_bytes
        need = size(M, E, d_out, d_in, dtype)
        call = lambda ws: [fn(tokens, c["offsets"], c["W_b"], c["B"], c["v"], axis, workspace=ws,
                              out=torch.full((M, width), 3.0, dtype=dtype, device=DEV))]
        if need > 0:
            in_exactly(need, call, call(None))


@pytest.mark.parametrize("axis", [ROW, COL])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("counts,d_out,d_in", [([9, 0, 70, 1], 2603, 2080), ([41] * 9, 1301, 1056), ([201], 515, 64), ([201, 3], 1032, 4128)])
def test_scale_gradient(counts, d_out, d_in, dtype, axis):
    c = make(counts, d_out, d_in, dtype, axis, 600 + d_out, before=2, behind=1)
    need = pd.pdelta_grad_v_experts_workspace_bytes(c["X"].shape[0], len(counts), d_out, d_in, axis)
    call = lambda ws: [pd.pdelta_grad_v_experts(c["X"], c["dY"], c["offsets"], c["B"], axis, workspace=ws)]
    in_exactly(need, call, call(None))


@pytest.mark.parametrize("T,V,k,dtype", [(3, 70001, 7, BF16), (5, 40001, 3, F32), (1, 152064, 1, F16), (127, 65601, 11, F16)])
def test_loss(T, V, k, dtype):
    logits, ids, top, _ = make_loss(T, V, k, dtype, V)
    need = pd.pdelta_distill_workspace_bytes(T, V, k, dtype)
    in_exactly(need, lambda ws: pd.pdelta_distill(logits, ids, top, workspace=ws), pd.pdelta_distill(logits, ids, top))


@pytest.mark.parametrize("axis", [ROW, COL])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("counts", [[1, 2], [9, 0, 5], [16, 11], [30, 31], [17, 3, 0, 40]])
def test_what_is_not_a_number_stays_in_its_row_of_few_tokens(counts, dtype, axis):
    c = make(counts, 96, 256, dtype, axis, 9, before=1, behind=2)
    n = c["X"].shape[0]
    clean = pd.pdelta_linear_experts(c["X"], c["offsets"], c["W_b"], c["B"], c["v"], axis)
    c["X"][1, 3], c["X"][3, 7], c["X"][0], c["X"][-2:] = float("nan"), float("inf"), float("nan"), float("nan")
    got = pd.pdelta_linear_experts(c["X"], c["offsets"], c["W_b"], c["B"], c["v"], axis)
    others = [m for m in range(1, n - 2) if m not in (1, 3)]
    assert torch.equal(got[others], clean[others])
    assert got[1].isnan().all() and not got[3].isfinite().any()
