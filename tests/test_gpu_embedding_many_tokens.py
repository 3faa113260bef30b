"""Embedding gradient of more tokens than one launch sorts (65536): digits sorted by two launches each, rows without tokens
cleared by the sums' launch.  Gradients of whole numbers are exact: their sums stay below 2^24."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def runner(*a, **kw):
    from paper_2505_05086_b200.runner import EmbeddingRunner
    return EmbeddingRunner(*a, **kw)


def world(V, D, T, dt, off=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T)
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * torch.log(torch.tensor(V + 1.0, dtype=torch.float64))).long() - 1).clamp(0, V - 1)
    flat = torch.zeros(off + T * D, device="cuda", dtype=dt)
    d = flat[off:].view(T, D)
    d.copy_(torch.randint(-8, 9, (T, D), generator=g, device="cuda").float())
    return ids, d, g


def plain(V, D, ids, d, scale, padding):
    keep = (ids >= 0) & (ids < V) & (ids != (padding if padding is not None else -1))
    return torch.zeros(V, D, device="cuda").index_add_(0, ids[keep], d[keep].float()) * scale


# one digit, two, three and four (odd and even numbers of passes), tiles of 8192 tokens met exactly and missed by one
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("V,D,T,off", [(200, 12, 65537, 0), (255, 3, 73728, 1), (256, 8, 73729, 0), (40000, 33, 100003, 3),
                                       (70000, 20, 131072, 0), (300, 770, 131071, 0), (1 << 24, 1, 70000, 0), (9000, 2056, 65600, 0)])
def test_gradient_of_whole_numbers_is_exact(V, D, T, off, dt):
    ids, d, g = world(V, D, T, dt, off)
    pad = int(ids[T // 2])
    ids[::11] = -3
    ids[5::17] = V + 4
    for padding in (None, pad):
        r = runner(V, D, T, bf16=dt == BF, scale=0.5, padding_idx=padding)
        want = plain(V, D, ids, d, 0.5, padding)
        dw = torch.full((off + V * D,), float("nan"), device="cuda")[off:].view(V, D)
        r.wgrad(ids, d, dw)
        assert torch.equal(dw, want)
        start = torch.randint(-99, 99, (V, D), generator=g, device="cuda").float()
        dw.copy_(start)
        r.wgrad(ids, d, dw, accumulate=True)
        assert torch.equal(dw, start + want)


def test_every_token_the_same_and_none_that_counts():
    V, D, T = 50, 24, 200000
    ids, d, _ = world(V, D, T, F32)
    r = runner(V, D, T, padding_idx=3)
    dw = torch.empty(V, D, device="cuda")
    for v in (0, 49, 3, -1, V):
        ids.fill_(v)
        dw.fill_(7)
        r.wgrad(ids, d, dw)
        assert torch.equal(dw, plain(V, D, ids, d, 1.0, 3))


def test_shorter_batches_in_the_workspace_of_a_longer_one():
    V, D = 3000, 40
    r = runner(V, D, 140000)
    dw = torch.empty(V, D, device="cuda")
    for T in (140000, 65537, 65536, 1025, 1024, 0, 90001):
        ids, d, _ = world(V, D, T, F32, seed=1)
        r.wgrad(ids, d, dw)
        assert torch.equal(dw, plain(V, D, ids, d, 1.0, None))


def test_same_bits_again_and_in_a_graph():
    V, D, T = 5000, 64, 100000
    ids, d, g = world(V, D, T, F32)
    d.copy_(torch.randn(T, D, generator=g, device="cuda"))
    r = runner(V, D, T)
    dw, other = torch.empty(V, D, device="cuda"), torch.empty(V, D, device="cuda")
    r.wgrad(ids, d, dw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.wgrad(ids, d, other)
    for _ in range(2):
        other.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, other)
    want = torch.zeros(V, D, device="cuda", dtype=torch.float64).index_add_(0, ids, d.double())
    size = torch.zeros(V, D, device="cuda", dtype=torch.float64).index_add_(0, ids, d.double().abs())
    # each addition rounds by half a step, 2^-24, of a partial sum that the sum of magnitudes bounds
    count = torch.bincount(ids, minlength=V)[:, None]
    assert ((dw.double() - want).abs() <= (count + 8) * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("T,D,hot", [(1 << 20, 3, 1.0), (1 << 20, 8, 0.6), (40000, 64, 1.0), (70001, 5, 0.3)])
def test_runs_over_hundreds_of_chunks(T, D, hot):
    """Where such a run starts and ends is found by a search, not chunk by chunk: between rarer ids, at either end, alone."""
    V = 900
    for v in (0, 450, V - 1):
        g = torch.Generator(device="cuda").manual_seed(v)
        ids = torch.randint(0, V, (T,), generator=g, device="cuda")
        ids[torch.rand(T, generator=g, device="cuda") < hot] = v
        d = torch.randint(-8, 9, (T, D), generator=g, device="cuda").float()
        r = runner(V, D, T)
        dw, want = torch.empty(V, D, device="cuda"), plain(V, D, ids, d, 1.0, None)
        r.wgrad(ids, d, dw)
        assert torch.equal(dw, want)
        r.wgrad(ids, d, dw, accumulate=True)
        assert torch.equal(dw, 2 * want)
