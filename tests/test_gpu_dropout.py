"""Dropout by the counter-based generator against its definition: the mask exactly, values to their last rounding."""
import numpy as np
import pytest
import torch

from tests.block_util import U16, U32, factors, half_words

pytestmark = pytest.mark.gpu
DT = {True: torch.bfloat16, False: torch.float32}


def close(got, want, size, bf16):
    """One product and one sum in fp32 (two half steps of what goes in), rounded once."""
    return ((got.double().cpu() - want).abs() <= 2 * U32 * size + (U16 if bf16 else U32) * want.abs()).all()


@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 100003])
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("res", [True, False])
def test_values_and_gradient(n, bf16, res):
    from paper_2505_05086_b200.runner import DropoutRunner
    g = torch.Generator(device="cuda").manual_seed(n)
    x, r = (torch.randn(n, generator=g, device="cuda").to(DT[bf16]) for _ in range(2))
    out = torch.full((n + 8,), 7.0, device="cuda", dtype=DT[bf16])
    op = DropoutRunner(0.3, seed=(5 << 40) + 11, stream_id=9, bf16=bf16)
    op.forward(x, out[:n], step=77, residual=r if res else None)
    f = factors(0.3, (5 << 40) + 11, 9, 77, n)
    want = x.double().cpu() * f + (r.double().cpu() if res else 0)
    assert close(out[:n], want, (x.double().cpu() * f).abs() + r.double().abs().cpu(), bf16)
    assert (out[n:] == 7).all()
    if not res:                                                       # the gradient is the same factors' product; in place too
        assert torch.equal(out[:n].cpu() == 0, f == 0)
        again = x.clone()
        op.backward(again, again, step=77)
        assert torch.equal(again, out[:n])


@pytest.mark.parametrize("p,kept", [(0.0, 1.0), (1e-6, 1.0), (0.5, 0.5), (1 - 2.0 ** -16, 2.0 ** -16)])
def test_probabilities(p, kept):
    from paper_2505_05086_b200.runner import DropoutRunner
    n = 1 << 20
    x, out = torch.ones(n, device="cuda"), torch.empty(n, device="cuda")
    DropoutRunner(p, seed=3).forward(x, out)
    assert torch.equal(out.cpu(), factors(p, 3, 0, 0, n).float())
    # sixteen bits a draw: the share stays within six deviations
    assert abs(float((out != 0).float().mean()) - kept) <= 6 * np.sqrt(kept * (1 - kept) / n)


def test_rows_off_their_alignment_and_steps_on_the_device():
    from paper_2505_05086_b200.runner import DropoutRunner
    for bf16 in (True, False):
        x = torch.randn(3001, device="cuda").to(DT[bf16])
        out = torch.zeros(3003, device="cuda", dtype=DT[bf16])
        op = DropoutRunner(0.2, seed=1, stream_id=4, bf16=bf16)
        step = torch.tensor([(1 << 32) + 6], device="cuda")          # (its low 32 bits count)
        op.forward(x[1:], out[2:3002], step=step)
        f = factors(0.2, 1, 4, 6, 3000)
        assert close(out[2:3002], x[1:].double().cpu() * f, x[1:].double().abs().cpu() * f, bf16)
        assert out[0] == out[1] == out[3002] == 0


def test_what_is_dropped_may_be_anything():
    from paper_2505_05086_b200.runner import DropoutRunner
    f = factors(0.5, 8, 0, 0, 4096)
    x = torch.where(f == 0, float("nan"), 1.0).float().cuda()
    x[::2] = torch.where(f[::2] == 0, float("inf"), 1.0).float().cuda()
    r, out = torch.ones(4096, device="cuda"), torch.empty(4096, device="cuda")
    DropoutRunner(0.5, seed=8).forward(x, out, residual=r)
    assert torch.equal(out.cpu(), f.float() + 1)
    x = torch.full((4096,), float("nan"), device="cuda")             # and what is kept stays what it is
    DropoutRunner(0.5, seed=8).forward(x, out)
    assert torch.equal(out.isnan().cpu(), f != 0)


def test_a_captured_step_draws_new_masks():
    from paper_2505_05086_b200.runner import DropoutRunner
    n = 5000
    x, out, step = torch.ones(n, device="cuda"), torch.empty(n, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    op = DropoutRunner(0.4, seed=2)
    op.forward(x, out, step=step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(x, out, step=step)
        step += 1
    for t in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), factors(0.4, 2, 0, t, n).float())


def test_far_elements():
    """More than 2^32 elements, in place: their places count in 64 bits."""
    from paper_2505_05086_b200.runner import DropoutRunner
    n = (1 << 32) + 4097
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    DropoutRunner(0.5, seed=6, bf16=True).forward(x, x)
    for first in (0, (1 << 31) - 1000, n - 5000):
        k = half_words(6, 0, 0, first, 5000) >= 32768
        assert torch.equal(x[first:first + 5000].cpu(), torch.from_numpy(k).to(torch.bfloat16) * 2)
