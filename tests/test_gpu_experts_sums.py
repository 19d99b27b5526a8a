"""GPU: the scale gradient's sums over a run of tiles stay as short as the bounds of experts_util say."""
import pytest
import torch

from experts_util import COL, ROW, U
from paper_2512_19720_amd import binding as pd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("axis", [ROW, COL])
def test_sums_over_many_tiles(axis):
    """One token for each of 16 experts, all products x = 0.9922 and all signs +1: a lane's sum of all 8 tiles would pass 256, where an
    addition of x loses 15/32 of a unit each time, 120 u = 120 2^-24 in all.  A term takes part in one product, 64 additions inside a
    tile, two between lanes and waves and 8 between tiles: 75 u."""
    E, kept, summed = 16, 4096, 2048
    a, b = 1.0 - 3 / 1024, 1.0 - 5 / 1024
    d_out, d_in = (kept, summed) if axis == ROW else (summed, kept)
    X = torch.full((E, d_in), a, dtype=torch.float16, device=DEV)
    dY = torch.full((E, d_out), b, dtype=torch.float16, device=DEV)
    offsets = torch.arange(E + 1, dtype=torch.int32, device=DEV)
    B = torch.full((E, d_out, d_in // 32), -1, dtype=torch.int32, device=DEV)
    got = pd.pdelta_grad_v_experts(X, dY, offsets, B, axis).double()
    want = a * b * summed
    off = float((got / want - 1).abs().max()) / U
    assert off <= 1 + 64 + 2 + summed / 256, off
