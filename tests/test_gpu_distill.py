"""GPU: the loss against a teacher's top logits and its gradient, against the 64-bit form of experts_util with its bounds."""
import pytest
import torch

from experts_util import distill64, distill_bounds, held
from paper_2512_19720_amd import binding as pd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def make(T, V, k, dtype, seed, top_dtype=None, scale=2.5):
    g = torch.Generator().manual_seed(seed)
    logits = (torch.randn(T, V, generator=g) * scale).to(dtype)
    top, ids = torch.topk(logits.float() + 0.7 * torch.randn(T, V, generator=g), min(k, V), dim=1)
    if k > V:                                         # more slots than words: the others are not in use
        ids = torch.cat([ids, torch.full((T, k - V), -1)], 1)
        top = torch.cat([top, torch.zeros(T, k - V)], 1)
    return logits.to(DEV), ids.to(torch.int32).to(DEV), top.to(top_dtype or dtype).to(DEV), g


def check(logits, ids, top, weight, temperature, grad_scale, what):
    loss, grad = pd.pdelta_distill(logits, ids, top, weight, temperature, grad_scale)
    ref_loss, ref_grad = distill64(logits, ids, top, weight, temperature, grad_scale)
    loss_bound, grad_bound = distill_bounds(logits, ids, top, weight, temperature, grad_scale)
    fine = torch.isfinite(ref_loss)
    assert torch.equal(torch.isfinite(loss.cpu()), fine) and (loss.cpu()[~fine] == ref_loss[~fine]).all(), what
    held(loss.cpu()[fine], ref_loss[fine], loss_bound[fine] + 1e-30, f"loss {what}")
    held(grad, ref_grad, grad_bound, f"grad {what}")
    alone, none = pd.pdelta_distill(logits, ids, top, weight, temperature, grad_scale, want_grad=False)
    assert none is None and torch.equal(alone, loss)
    place = logits.clone()
    loss2, grad2 = pd.pdelta_distill(place, ids, top, weight, temperature, grad_scale, out=place)
    assert grad2 is place and torch.equal(place, grad) and torch.equal(loss2, loss)
    return loss, grad


# one word, vocabularies around vectors, waves and workgroups, odd ones (rows at every alignment), large ones
SIZES = [(1, 1, 1), (3, 2, 2), (5, 7, 3), (4, 64, 64), (9, 1000, 16), (33, 1023, 5), (8, 4099, 100), (2, 32001, 8), (3, 70001, 1024), (1, 152064, 20)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("T,V,k", SIZES)
def test_loss_and_gradient_match(T, V, k, dtype):
    logits, ids, top, _ = make(T, V, k, dtype, T + V)
    check(logits, ids, top, None, 1.0, 256.0 if dtype == F16 else 1.0, f"{T}x{V} k {k} {dtype}")


@pytest.mark.parametrize("T", [1, 17, 300, 1000])
def test_number_of_tokens(T):
    logits, ids, top, _ = make(T, 2051, 6, BF16, T)
    check(logits, ids, top, None, 1.0, 1.0, f"{T} tokens")


@pytest.mark.parametrize("temperature", [0.05, 0.7, 1.0, 2.0, 40.0])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_temperatures_with_masked_words(temperature, dtype):
    logits, ids, top, _ = make(6, 3001, 12, dtype, 3)
    logits[:, 2900:] = float("-inf")
    ids = torch.where(ids < 2900, ids, -1)
    check(logits, ids, top, None, temperature, 3.0, f"temperature {temperature}")


@pytest.mark.parametrize("top_dtype", [F32, F16, BF16])
def test_types_of_the_teacher(top_dtype):
    logits, ids, top, _ = make(6, 500, 9, BF16, 4, top_dtype)
    check(logits, ids, top, None, 1.0, 1.0, f"teacher in {top_dtype}")


def test_slots_words_and_weights():
    logits, ids, top, g = make(9, 777, 10, F32, 5)
    ids[0] = -1                                       # no slot in use
    ids[1, 3:] = 777                                  # behind the vocabulary
    ids[2, :] = ids[2, 0]                             # one word in every slot
    ids[3, 5] = ids[3, 4]                             # one word twice
    top[4, 1:] = float("-inf")                        # one share of 1
    top[5] = torch.finfo(torch.float32).min           # equal shares
    ids[6, 2] = -2 ** 31
    weight = torch.tensor([1.0, 0.5, 2.0, 1.0, 1e-3, 1.0, 1.0, 0.0, -1.0], device=DEV)
    logits[7] = float("nan")                          # weight 0: whatever the logits are
    clean = logits.clone()
    clean[7] = 0
    loss, grad = pd.pdelta_distill(logits, ids, top, weight, 1.5, 4.0)
    ref_loss, ref_grad = distill64(clean, ids, top, weight, 1.5, 4.0)
    loss_bound, grad_bound = distill_bounds(clean, ids, top, weight, 1.5, 4.0)
    held(loss, ref_loss, loss_bound + 1e-30, "loss")
    held(grad, ref_grad, grad_bound, "grad")
    assert float(loss[0]) == 0 and not grad[0].any() and float(loss[7]) == 0 and not grad[7].any()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_masked_words_and_rows(dtype):
    logits, ids, top, _ = make(5, 300, 4, dtype, 6)
    logits[0, ids[0, 1].long()] = float("-inf")       # the teacher answers with a masked word
    logits[1] = float("-inf")                         # nothing may be answered
    logits[2, 1:] = float("-inf")                     # one word may
    ids[2] = torch.tensor([0, -1, -1, -1], dtype=torch.int32)
    lowest = torch.finfo(dtype).min
    logits[3, 5:] = lowest                            # a mask of the type's lowest value
    ids[3] = torch.tensor([0, 1, 2, 3], dtype=torch.int32)
    loss, grad = pd.pdelta_distill(logits, ids, top)
    ref_loss, ref_grad = distill64(logits, ids, top, None, 1.0, 1.0)
    assert loss[0] == float("inf") and loss[1] == float("inf")
    assert grad.isfinite().all() and not grad[2].any() and float(loss[2]) == 0
    easy = torch.where(logits < -1e4, torch.tensor(-50.0, dtype=dtype, device=DEV), logits)
    loss_bound, grad_bound = distill_bounds(easy, ids, top, None, 1.0, 1.0)
    held(loss[2:], ref_loss[2:], loss_bound[2:], "loss")
    held(grad, ref_grad, grad_bound, "grad")


def test_no_tokens():
    loss, grad = pd.pdelta_distill(torch.empty(0, 50, dtype=BF16, device=DEV), torch.empty(0, 3, dtype=torch.int32, device=DEV),
                                   torch.empty(0, 3, dtype=BF16, device=DEV))
    assert loss.shape == (0,) and grad.shape == (0, 50)


@pytest.mark.parametrize("T,V", [(2, 50001), (700, 1003)])
def test_captured_and_on_another_stream(T, V):
    logits, ids, top, _ = make(T, V, 8, BF16, 7)
    weight = torch.ones(T, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        aside = pd.pdelta_distill(logits, ids, top, weight)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pd.pdelta_distill(logits, ids, top, weight)
    for k in range(4):
        fresh = make(T, V, 8, BF16, 7 + k)
        for a, b in zip((logits, ids, top), fresh):
            a.copy_(b)
        weight[k % T] = 0.0
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = pd.pdelta_distill(logits, ids, top, weight)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        if k == 0:
            weight.fill_(1.0)
            assert all(torch.equal(a, b) for a, b in zip(aside, pd.pdelta_distill(logits, ids, top, weight)))


def test_rows_behind_two_to_the_31():
    """Entries whose place in the matrix passes 31 bits: the last rows of a call like those of a call of their own."""
    T, V = 16600, 131072
    logits = torch.zeros(T, V, dtype=BF16, device=DEV)
    rest, ids_rest, top_rest, _ = make(3, V, 8, BF16, 9)
    logits[-3:] = rest
    ids, top = torch.full((T, 8), -1, dtype=torch.int32, device=DEV), torch.zeros(T, 8, dtype=BF16, device=DEV)
    ids[-3:], top[-3:] = ids_rest, top_rest
    loss, grad = pd.pdelta_distill(logits, ids, top, out=logits)
    want_loss, want_grad = pd.pdelta_distill(rest, ids_rest, top_rest)
    assert not loss[:-3].any() and not grad[:100].any() and not grad[8000:8100].any()
    loss_bound, grad_bound = distill_bounds(rest, ids_rest, top_rest, None, 1.0, 1.0)
    held(loss[-3:], want_loss.cpu().double(), 2 * loss_bound, "loss")
    held(grad[-3:], want_grad.cpu().double(), 2 * grad_bound, "grad")


# rows that end at and behind what a workgroup keeps in registers, of more tokens than are split among workgroups
@pytest.mark.parametrize("T,V,dtype", [(130, 16384, F16), (5, 16385, BF16), (40, 16399, F16), (129, 32769, BF16), (131, 65536, F16), (129, 65601, F16),
                                       (130, 70001, BF16), (129, 81927, F16), (129, 81928, BF16), (129, 131099, F16), (129, 8192, F32), (3, 8196, F32),
                                       (129, 40963, F32), (130, 40964, F32), (129, 98304, BF16), (129, 98313, F16), (129, 49159, F32)])
def test_rows_longer_than_what_is_kept(T, V, dtype):
    logits, ids, top, g = make(T, V, 12, dtype, T + V)
    logits[1::3, V // 2:] = float("-inf")
    logits[2::5, :V - 3] = -60000.0                   # the largest of the row in its last words
    top[logits.gather(1, ids.long()).isinf()] = float("-inf")
    weight = torch.rand(T, generator=g).to(DEV)
    weight[::7] = 0
    check(logits, ids, top, weight, 1.3, 2.0, f"{T}x{V} {dtype}")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("peak", [5.0, 20.0, 27.0, 29.0, 60.0, 500.0])
def test_words_far_above_the_others(peak, dtype):
    """A word e^peak above the rest, at every place that a wave may meet it first or last; some of them stand before masked words."""
    T, V = 48, 12345
    logits, ids, top, g = make(T, V, 8, dtype, int(peak), scale=0.3)
    at = torch.linspace(0, V - 1, T).long()
    logits[torch.arange(T), at] = peak
    logits[::4, :4096] = float("-inf")
    ids[:, 0] = at.to(torch.int32).to(DEV)
    top[logits.gather(1, ids.long()).isinf()] = float("-inf")
    check(logits, ids, top, None, 1.0, 1.0, f"peak {peak} {dtype}")
