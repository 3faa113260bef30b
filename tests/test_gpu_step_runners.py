"""Runners of the token loss, embedding and AdamW on streams other than the one their buffers were made on."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def busy(block, fills=50):
    """Queues work on the current stream that goes on writing to `block`."""
    big = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for _ in range(fills):
        big.fill_(1)
        block.fill_(255)
    return big


def test_first_gradient_on_another_stream_while_the_memory_is_still_in_use():
    """The workspace lies where the current stream still writes: the other stream waits for it."""
    from paper_2505_05086_b200.runner import EmbeddingRunner
    V, D, T = 900, 64, 3000
    g = torch.Generator(device="cuda").manual_seed(0)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    d = torch.randint(-8, 9, (T, D), generator=g, device="cuda").float()
    want = torch.zeros(V, D, device="cuda").index_add_(0, ids, d)
    dw = torch.empty(V, D, device="cuda")
    size = EmbeddingRunner(V, D, T).ws.numel()
    side = torch.cuda.Stream()
    for _ in range(3):
        block = torch.empty(size, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        keep, at = busy(block), block.data_ptr()
        del block
        r = EmbeddingRunner(V, D, T)
        assert r.ws.data_ptr() == at
        r.wgrad(ids, d, dw, stream=side)
        side.synchronize()
        assert torch.equal(dw, want)
        del r, keep


def test_a_dropped_runner_keeps_its_memory_until_the_other_stream_is_done():
    from paper_2505_05086_b200.runner import EmbeddingRunner
    V, D, T = 900, 64, 3000
    ids, d, dw = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.ones(T, D, device="cuda"), torch.empty(V, D, device="cuda")
    side = torch.cuda.Stream()
    r = EmbeddingRunner(V, D, T)
    size, at = r.ws.numel(), r.ws.data_ptr()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        keep = busy(torch.empty(16, dtype=torch.uint8, device="cuda"))
        r.wgrad(ids, d, dw)
    del r
    other = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert other.data_ptr() != at
    other.fill_(255)
    side.synchronize()
    assert (dw[0] == T).all() and (dw[1:] == 0).all()
    del keep


def test_results_on_another_stream_come_behind_what_cleared_them():
    from paper_2505_05086_b200.runner import LogprobRunner
    x, y = torch.zeros(64, 100, device="cuda"), torch.zeros(64, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = busy(torch.empty(16, dtype=torch.uint8, device="cuda"))
    r = LogprobRunner(64, 100)
    r.forward(x, y, stream=side)
    torch.cuda.synchronize()
    assert (r.logp < -4).all() and (r.lse > 4).all()
    del keep


def test_gradients_of_micro_batches_from_their_own_forward_pass():
    """Weights that come after several forward passes: each gradient goes by the lse and entropy of its own batch."""
    from paper_2505_05086_b200.runner import LogprobRunner
    T, V = 37, 500
    g = torch.Generator(device="cuda").manual_seed(1)
    batches = [(torch.randn(n, V, generator=g, device="cuda"), torch.randint(0, V, (n,), generator=g, device="cuda")) for n in (T, T - 8)]
    w = torch.randn(T, generator=g, device="cuda")
    want = []
    for x, y in batches:
        r, out = LogprobRunner(T, V), torch.empty_like(x)
        r.forward(x, y)
        r.backward(x, y, w[:len(y)], w[:len(y)], out)
        want.append(out)
    r, kept = LogprobRunner(T, V), []
    for x, y in batches:
        r.forward(x, y)
        kept.append((r.lse[:len(y)].clone(), r.entropy[:len(y)].clone()))
    for (x, y), (lse, entropy), right in zip(batches, kept, want):
        n, out = len(y), torch.empty_like(x)
        r.backward(x, y, w[:n], w[:n], out, lse=lse, entropy=entropy)
        assert torch.equal(out, right)
        r.lse, r.entropy = lse, entropy                              # or in place of the runner's own
        out.zero_()
        r.backward(x, y, w[:n], w[:n], out)
        assert torch.equal(out, right)
    fresh = torch.full((T,), 9.0, device="cuda")
    r.lse, r.entropy = fresh, torch.empty(T, device="cuda")
    r.forward(*batches[0])
    assert torch.equal(fresh, kept[0][0])


@pytest.mark.parametrize("bits8", [False, True])
def test_steps_behind_an_exchange_of_memory(bits8):
    """The same bits as a runner that was made with the new memory, and nothing in the old."""
    from paper_2505_05086_b200.runner import AdamWRunner
    g = torch.Generator(device="cuda").manual_seed(2)
    ws, gs = ([torch.randn(n, generator=g, device="cuda") for n in (3000, 5)] for _ in range(2))
    a = AdamWRunner([w.clone() for w in ws], [x.clone() for x in gs], bits8=bits8)
    b = AdamWRunner([w.clone() for w in ws], [x.clone() for x in gs], bits8=bits8)
    a.step(), b.step()
    old = [w.detach() for w in b.weights]
    before = [w.clone() for w in old]
    for w, x in zip(b.weights, b.grads):
        w.data, x.data = w.data.clone(), x.data.clone()
    a.step(), b.step()
    assert all(torch.equal(x, y) for x, y in zip(a.weights, b.weights))
    assert all(torch.equal(x, y) for x, y in zip(old, before))
