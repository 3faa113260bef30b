"""What the output layer's gradients are held to beyond their elementwise bounds, each by a quantity of its own."""
import pytest
import torch

from tests.test_gpu_head import World

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16_dw", [True, False, None])
@pytest.mark.parametrize("T,V,D", [(9, 9000, 264), (300, 4000, 136), (1500, 32000, 128), (2100, 3000, 136), (2100, 2500, 75)])
def test_dx_gets_back_what_rounding_takes_from_g_at_the_target(T, V, D, bf16_dw):
    """G's target entry is scale dlogp (1 - p); without the remainder off_t that its rounding to bf16 takes, dx is off by -off_t w[y_t].  So the error of dx is
    projected on that: -1 without the remainder, 0 with it, give or take what else is rounded.  That is dx itself (half a step, 2^-8 of a value at
    most, of random sign) and G's other entries (p_j, whose roundings reach dx as sums over w): a rounding of dx is below 3/2 max |off| |w| in the mean
    square where off is uniform within its step, and T D >= 2376 elements average it down to 0.06 at most.  A quarter is four of those."""
    w = World(T, V, D, bf16=True, bf16_dw=bool(bf16_dw), scale=0.7)
    got = w.loss(dw=bf16_dw is not None)
    r = w.reference()
    live = w.y != -100
    hot = r["G"][torch.arange(T, device="cuda"), w.y.clamp(min=0)]
    off = torch.where(live, hot - hot.float().bfloat16().double(), 0.0)
    lost = off[:, None] * w.w[w.y.clamp(min=0)].double()
    share = float(((got["dx"].double() - r["dx"]) * lost).sum() / lost.square().sum())
    assert abs(share) <= 0.25
