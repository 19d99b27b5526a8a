"""GPU: the loss against a teacher's top logits where a teacher's or a student's logit is no finite number."""
import pytest
import torch

from paper_2512_19720_amd import binding as pd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")

# rows of one workgroup, with all of it in registers and with more, and (few long ones) rows that are split among workgroups
SIZES = [(6, 77, 1, F32), (6, 777, 5, F16), (200, 20003, 9, BF16), (131, 65601, 3, F32), (3, 70001, 7, BF16), (5, 40001, 4, F32), (2, 152064, 3, F16)]


def make(T, V, k, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    logits = (torch.randn(T, V, generator=g, device=DEV) * 2.5).to(dtype)
    top, ids = torch.topk(logits.float(), k, dim=1)
    return logits, ids.to(torch.int32), (top + 0.5 * torch.randn(T, k, generator=g, device=DEV)).to(dtype)


def every_form(logits, ids, top, weight=None):
    """(loss, gradient), the same from the loss alone and from the gradient in the logits' place."""
    loss, grad = pd.pdelta_distill(logits, ids, top, weight, 1.5, 4.0)
    alone, _ = pd.pdelta_distill(logits, ids, top, weight, 1.5, 4.0, want_grad=False)
    place = logits.clone()
    loss2, grad2 = pd.pdelta_distill(place, ids, top, weight, 1.5, 4.0, out=place)
    for a, b in ((alone, loss), (loss2, loss), (grad2, grad)):
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0), b.nan_to_num(0))
    return loss, grad


def others_alike(got, clean, rows):
    keep = torch.ones(got.shape[0], dtype=torch.bool, device=DEV)
    keep[rows] = False
    assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("T,V,k,dtype", SIZES)
def test_a_teachers_logit_that_is_no_number(T, V, k, dtype):
    """softmax of the row's top logits is NaN for every slot: the loss is, and the gradient at their words; the rest is q."""
    logits, ids, top = make(T, V, k, dtype, V)
    clean_loss, clean_grad = every_form(logits, ids, top)
    for bad in (NAN, INF):
        for slots in ([0], [k - 1], list(range(k))):
            wrong = top.clone()
            wrong[1, slots] = bad
            loss, grad = every_form(logits, ids, wrong)
            assert loss[1].isnan(), (bad, slots)
            words = torch.zeros(V, dtype=torch.bool, device=DEV)
            words[ids[1].long()] = True
            assert grad[1, words].isnan().all() and torch.equal(grad[1, ~words], clean_grad[1, ~words]), (bad, slots)
            others_alike(loss, clean_loss, [1])
            others_alike(grad, clean_grad, [1])
    # what is not in use does not matter, whatever it holds
    if k > 1:
        unused, plain = ids.clone(), top.clone()
        unused[:, -1] = -1
        plain[:, -1] = NAN
        loss, grad = every_form(logits, unused, plain)
        assert loss.isfinite().all() and grad.isfinite().all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("bits", [0x7FFFFFFF, -1, 0x7FC00000, 0x7F800001])
def test_a_teachers_nan_of_any_pattern(bits, dtype):
    logits, ids, top = make(3, 501, 4, dtype, 2)
    top = top.float()
    top.view(torch.int32)[1, 2] = bits
    loss, grad = every_form(logits, ids, top)
    assert loss[1].isnan() and grad[1, ids[1].long()].isnan().all() and loss[[0, 2]].isfinite().all() and grad[[0, 2]].isfinite().all()


@pytest.mark.parametrize("T,V,k,dtype", SIZES)
def test_a_students_logit_that_is_no_number(T, V, k, dtype):
    """softmax over the vocabulary is NaN for every word: the loss is, and the row of the gradient."""
    logits, ids, top = make(T, V, k, dtype, V + 1)
    clean_loss, clean_grad = every_form(logits, ids, top)
    for bad in (NAN, INF):
        for at in (0, 1, V // 2, V - 1, slice(V // 3, V // 3 + 9), slice(None)):
            wrong = logits.clone()
            wrong[1, at] = bad
            loss, grad = every_form(wrong, ids, top)
            assert loss[1].isnan() and grad[1].isnan().all(), (bad, at)
            others_alike(loss, clean_loss, [1])
            others_alike(grad, clean_grad, [1])
        # nothing else may be answered
        wrong = logits.clone()
        wrong[1] = -INF
        wrong[1, 2 * V // 3] = bad
        loss, grad = every_form(wrong, ids, top)
        assert loss[1].isnan() and grad[1].isnan().all(), bad
        others_alike(grad, clean_grad, [1])


@pytest.mark.parametrize("T,V,k,dtype", SIZES)
def test_a_token_without_a_slot_in_use(T, V, k, dtype):
    """Loss and gradient are 0 whatever the token's logits hold: the rows of padding of a batch."""
    logits, ids, top = make(T, V, k, dtype, V + 2)
    clean_loss, clean_grad = every_form(logits, ids, top)
    ids[1] = -1
    for row in (1, 0):
        if row == 0:
            top[0] = -INF                             # slots, but no share
        for bad in (NAN, INF, -INF):
            for at in (V // 2, slice(None)):
                wrong = logits.clone()
                wrong[row, at] = bad
                loss, grad = every_form(wrong, ids, top)
                assert float(loss[row]) == 0 and not grad[row].any(), (row, bad, at)
                others_alike(loss, clean_loss, [0, 1])
                others_alike(grad, clean_grad, [0, 1])
