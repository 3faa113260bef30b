"""Calls of the token loss that the documentation allows and that are easily forgotten."""
import pytest
import torch

pytestmark = pytest.mark.gpu
IGN = -100


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_results_between_the_rows_of_logits_and_gradient(dt):
    """Buffers that lie whole behind a row, through the binding: neither refused nor written over."""
    from paper_2505_05086_b200 import binding as B
    T, V, gap = 5, 70, 42
    g = torch.Generator(device="cuda").manual_seed(0)
    e = torch.finfo(dt).bits // 8
    x = torch.full((T, V + gap), 7.0, device="cuda", dtype=dt)
    x[:, :V] = torch.randn(T, V, generator=g, device="cuda")
    y, w = torch.randint(0, V, (T,), generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
    dx = torch.full_like(x, 7.0)
    s = torch.cuda.current_stream().cuda_stream
    d = B.LogprobDesc(1 if e == 2 else 0, 0, T, V, V + gap, V + gap, IGN, 1.0)
    logp, ent, lse = (torch.empty(T, device="cuda") for _ in range(3))
    want = torch.empty_like(x)
    B.token_loss(d, x.data_ptr(), y.data_ptr(), w.data_ptr(), w.data_ptr(), logp.data_ptr(), ent.data_ptr(), lse.data_ptr(), want.data_ptr(), s)
    at_x = x.data_ptr() + (V + gap + V + 2) * e                      # behind the second row: 20 bytes each, on 4
    at_dx = dx.data_ptr() + (2 * (V + gap) + V + 2) * e
    B.token_loss(d, x.data_ptr(), y.data_ptr(), w.data_ptr(), w.data_ptr(), at_x, at_x + 20, at_dx, dx.data_ptr(), s)
    torch.cuda.synchronize()
    assert torch.equal(dx[:, :V], want[:, :V])
    behind = x[1, V + 2:V + 2 + 40 // e].view(torch.uint8).view(torch.float32)
    assert torch.equal(behind, torch.cat([logp, ent]))
    assert torch.equal(dx[2, V + 2:V + 2 + 20 // e].view(torch.uint8).view(torch.float32), lse)
    assert (x[0, V:] == 7).all() and (dx[0, V:] == 7).all() and (dx[3:, V:] == 7).all()
