"""Offsets beyond 2^31 elements: rows of logits far apart, a large embedding, a tensor of more than 2^31 values."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def test_rows_of_logits_far_apart():
    from paper_2505_05086_b200.runner import LogprobRunner
    V, ld = 1003, 1_200_000_001
    flat = torch.empty(2 * ld + V, device="cuda", dtype=torch.bfloat16)
    x = flat.as_strided((3, V), (ld, 1))
    g = torch.Generator(device="cuda").manual_seed(0)
    # (rows that start at the same places within 16 bytes: the order of sums goes by that)
    near = torch.randn(3, 1009, generator=g, device="cuda").bfloat16()[:, :V]
    x.copy_(near)
    y, a = torch.tensor([5, 1002, 0], device="cuda"), torch.tensor([1.0, -2.0, 0.5], device="cuda")
    far, ref = LogprobRunner(3, V, bf16=True, top_k=7), LogprobRunner(3, V, bf16=True, top_k=7)
    far.forward(x, y), ref.forward(near, y)
    for name in ("logp", "lse", "entropy", "top_logp", "top_ids"):
        assert torch.equal(getattr(far, name), getattr(ref, name)), name
    out = torch.empty(3, V, device="cuda", dtype=torch.bfloat16)
    for form in ("backward", "loss"):
        getattr(ref, form)(near, y, a, a, out)
        getattr(far, form)(x, y, a, a, x)                            # in place
        assert torch.equal(x, out), form
        x.copy_(near)


def test_a_large_embedding():
    from paper_2505_05086_b200.runner import EmbeddingRunner
    V, D, T = 1_100_000, 2048, 500
    g = torch.Generator(device="cuda").manual_seed(0)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    ids[:3] = torch.tensor([V - 1, V - 1, 0], device="cuda")
    table = torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)
    table[ids] = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    r = EmbeddingRunner(V, D, T, bf16=True, bf16_table=True, scale=0.5)
    out = torch.empty(T, D, device="cuda", dtype=torch.bfloat16)
    r.forward(table, ids, out)
    assert torch.equal(out, (table[ids].float() * 0.5).bfloat16())
    del table
    torch.cuda.empty_cache()
    d = torch.randint(-8, 9, (T, D), generator=g, device="cuda").bfloat16()
    rows, where = torch.unique(ids, return_inverse=True)
    want = torch.zeros(len(rows), D, device="cuda").index_add_(0, where, d.float()) * 0.5
    dw = torch.full((V, D), 3.0, device="cuda")
    r.wgrad(ids, d, dw, accumulate=True)
    assert torch.equal(dw[rows], want + 3)
    r.wgrad(ids, d, dw)
    assert torch.equal(dw[rows], want)
    dw[rows] = 0
    assert all(not part.any() for part in dw.split(100_000))


def test_a_tensor_of_more_than_two_to_the_31_values():
    from paper_2505_05086_b200.runner import AdamWRunner
    n, tail = (1 << 31) + 300, 256 * 9 + 300 % 256                   # the tail starts on a block
    bf = dict(device="cuda", dtype=torch.bfloat16)
    w, g = torch.zeros(n, **bf), torch.zeros(n, **bf)
    gen = torch.Generator(device="cuda").manual_seed(0)
    w[-tail:], g[-tail:] = torch.randn(tail, generator=gen, device="cuda"), torch.randn(tail, generator=gen, device="cuda")
    w[:1000], g[:1000] = w[-1000:], g[-1000:]
    small = AdamWRunner([w[-tail:].clone()], [g[-tail:].clone()], bits8=True)
    large = AdamWRunner([w], [g], bits8=True)
    for _ in range(2):
        small.step(lr=0.01), large.step(lr=0.01)
    assert torch.equal(w[-tail:], small.weights[0])
    assert torch.equal(large.exp_avg[0][-tail:].view(torch.uint8), small.exp_avg[0].view(torch.uint8))
    assert torch.equal(large.exp_avg_sq[0][-tail:].view(torch.uint8), small.exp_avg_sq[0].view(torch.uint8))
    blocks = len(small.exp_avg_scale[0])
    assert torch.equal(large.exp_avg_scale[0][-blocks:].view(torch.uint8), small.exp_avg_scale[0].view(torch.uint8))
    assert all(not part.any() for part in w[1000:-tail].split(1 << 28))
