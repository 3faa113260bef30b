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


@pytest.mark.parametrize("T,V,off", [(5, 300, 1), (3, 50257, 0), (700, 1001, 0), (2, 131073, 3)])
@pytest.mark.parametrize("level", [150.0, -700.0, 1000.0, 3900.0])
def test_fp32_gradients_of_rows_off_zero_keep_their_digits(level, T, V, off):
    """An offset that all logits of a row share changes nothing about its gradient: from lse, which says little about differences
    there, it is as near to the definition as the loss in one pass (the same tolerance, which knows no |lse|)."""
    from tests.test_gpu_token_loss import check_grad, definition, make, runner
    x, y, _ = make(T, V, torch.float32, 5, off, seed=13)
    x += level
    y[0] = IGN
    alpha, beta = torch.linspace(0.5, 2, T, device="cuda"), torch.linspace(-1, 1, T, device="cuda")
    run = runner(T, V, torch.float32)
    run.forward(x, y)
    D = definition(x, y, 1.0)
    for b in (None, beta):
        out = torch.full((T, V + 5), 7.0, device="cuda")
        run.backward(x, y, alpha, b, out[:, :V])
        check_grad(out[:, :V], D, y, V, 1.0, alpha, b, torch.float32)
        assert (out[:, V:] == 7).all()
        again = x.clone()
        run.backward(again, y, alpha, b, again)                      # in place, in rows of another stride
        check_grad(again, D, y, V, 1.0, alpha, b, torch.float32)


@pytest.mark.parametrize("T", [3, 700])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scaled_logits_beyond_the_range_of_fp32(sign, T):
    """lse is infinite; all that goes by differences of logits stays what it is."""
    from tests.test_gpu_token_loss import runner
    V, scale = 50, 2.0 ** 26                                          # differences that the scale leaves exact
    g = torch.Generator(device="cuda").manual_seed(3)
    k = torch.randint(0, 4, (T, V), generator=g, device="cuda").float()
    level = sign * 2.0 ** 120
    x = torch.where(k > 0, level, level - 2.0 ** 100)                 # level, or so far below that nothing is left of it
    x[:, 0] = level
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    run = runner(T, V, torch.float32, scale=scale, top_k=5)
    run.forward(x, y)
    lead = x == level
    n = lead.sum(1)
    assert (run.lse == sign * float("inf")).all()
    hit = lead.gather(1, y[:, None])[:, 0]
    # log of a whole number up to 50 and its product with 1: a few roundings of 2^-24 of values up to 4
    assert ((run.entropy.double() - torch.log(n.double())).abs() <= 32 * 2.0 ** -24).all()
    assert ((run.logp.double() + torch.log(n.double())).abs() <= 32 * 2.0 ** -24)[hit].all()
    assert (run.logp[~hit] == -(2.0 ** 126)).all()                   # 2^26 times 2^100; log n is far below its last place
    v, i = torch.sort(x, dim=1, descending=True, stable=True)
    assert torch.equal(run.top_ids, i[:, :5])
    alpha = torch.randn(T, generator=g, device="cuda")
    want = scale * alpha[:, None].double() * (torch.zeros(T, V, device="cuda", dtype=torch.float64).scatter_(1, y[:, None], 1.0)
                                              - lead / n[:, None].double())
    for form in ("backward", "loss"):
        out = torch.empty_like(x)
        getattr(run, form)(x, y, alpha, None, out)
        assert ((out.double() - want).abs() <= 32 * 2.0 ** -24 * scale * alpha.abs()[:, None]).all()
