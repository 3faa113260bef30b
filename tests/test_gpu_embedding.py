"""Embedding lookup and its weight gradient.  Gradients of small whole numbers are exact in fp32 in any order (sums below
2^24), so those are compared for equality; others with (c + 8) u sum|terms| for c terms, u = 2^-24."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def runner(V, D, T, **kw):
    from paper_2505_05086_b200.runner import EmbeddingRunner
    return EmbeddingRunner(V, D, T, **kw)


def shifted(shape, dt, off):
    """A contiguous tensor that starts `off` elements behind an aligned address."""
    n = 1
    for s in shape:
        n *= s
    return torch.zeros(off + n + 8, device="cuda", dtype=dt)[off:off + n].view(shape)


@pytest.mark.parametrize("tt", [F32, BF])
@pytest.mark.parametrize("to", [F32, BF])
@pytest.mark.parametrize("V,D,T,off", [(1, 1, 1, 0), (7, 3, 5, 1), (100, 64, 33, 0), (100, 64, 33, 1), (50, 770, 20, 0),
                                       (333, 2048, 700, 0), (200, 36, 9, 4), (9, 5000, 3, 0)])
def test_lookup(V, D, T, off, tt, to):
    g = torch.Generator(device="cuda").manual_seed(V)
    table = shifted((V, D), tt, off)
    table.copy_(torch.randn(V, D, generator=g, device="cuda"))
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    out = shifted((T, D), to, off)
    scale = 45.254833995939045
    runner(V, D, T, bf16=to == BF, bf16_table=tt == BF, scale=scale).forward(table, ids, out)
    want = (table[ids].float() * torch.tensor(scale, dtype=F32)).to(to)      # one product, one rounding: the same bits
    assert torch.equal(out, want)


def test_lookup_of_ids_outside_the_vocabulary_and_of_shaped_ids():
    table = torch.ones(10, 8, device="cuda")
    ids = torch.tensor([[3, -1, 10], [0, 9, 1 << 40]], device="cuda")
    out = torch.zeros(2, 3, 8, device="cuda")
    r = runner(10, 8, 6)
    r.forward(table, ids, out)
    bad = torch.tensor([[False, True, True], [False, False, True]], device="cuda")
    assert torch.isnan(out[bad]).all() and (out[~bad] == 1).all()
    r.forward(table, ids[:0], out[:0])                                       # nothing to do


def zipf(T, V, g):
    return (torch.exp(torch.rand(T, generator=g, device="cuda") * torch.log(torch.tensor(V + 1.0))).long() - 1).clamp(0, V - 1)


SIZES = [(1, 1, 1, 0), (5, 3, 7, 1), (300, 8, 64, 0), (300, 64, 129, 4), (1000, 770, 2048, 0), (255, 40, 4096, 0),
         (256, 40, 5000, 0), (32000, 64, 4097, 0), (1025, 2056, 900, 0), (70000, 24, 20000, 0), (3, 48, 30000, 0),
         (1 << 21, 4, 3000, 0), (2000, 6000, 50, 0), (40000, 33, 9973, 3),
         (600, 20, 1024, 0), (600, 20, 1025, 0), (70000, 5, 1023, 1),
         (1 << 24, 1, 5000, 0), (65535, 12, 6000, 0), (65536, 12, 6000, 0), ((1 << 24) - 1, 2, 50000, 0), (70000, 3, 65536, 0)]


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("V,D,T,off", SIZES)
def test_gradient_of_whole_numbers_is_exact(V, D, T, off, dt):
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = zipf(T, V, g)
    d = shifted((T, D), dt, off)
    d.copy_(torch.randint(-8, 9, (T, D), generator=g, device="cuda").float())
    pad = int(ids[T // 2])
    ids[::11] = -3
    ids[5::17] = V + 4
    for padding in (None, pad):
        r = runner(V, D, T, bf16=dt == BF, scale=0.5, padding_idx=padding)
        keep = (ids >= 0) & (ids < V) & (ids != (pad if padding is not None else -1))
        want = torch.zeros(V, D, device="cuda").index_add_(0, ids[keep], d[keep].float()) * 0.5
        dw = shifted((V, D), F32, off)
        dw.fill_(float("nan"))
        r.wgrad(ids, d, dw)
        assert torch.equal(dw, want)
        start = torch.randint(-99, 99, (V, D), generator=g, device="cuda").float()
        dw.copy_(start)
        r.wgrad(ids, d, dw, accumulate=True)
        assert torch.equal(dw, start + want)


@pytest.mark.parametrize("T,hot", [(3000, 1.0), (30000, 1.0), (30000, 0.5), (700, 0.9)])
def test_frequent_ids_and_rounding(T, hot):
    """One id holds most tokens, or all: its run crosses many chunks."""
    V, D = 5000, 100
    g = torch.Generator(device="cuda").manual_seed(int(T * hot))
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    ids[torch.rand(T, generator=g, device="cuda") < hot] = 77
    d = torch.randn(T, D, generator=g, device="cuda")
    r = runner(V, D, T)
    dw, again = torch.empty(V, D, device="cuda"), torch.empty(V, D, device="cuda")
    r.wgrad(ids, d, dw)
    want = torch.zeros(V, D, device="cuda", dtype=torch.float64).index_add_(0, ids, d.double())
    size = torch.zeros(V, D, device="cuda", dtype=torch.float64).index_add_(0, ids, d.double().abs())
    count = torch.bincount(ids, minlength=V)[:, None]
    assert ((dw.double() - want).abs() <= (count + 8) * 2.0 ** -24 * size).all()
    r.wgrad(ids, d, again)
    assert torch.equal(dw, again)


def test_infinite_terms_stay_in_their_row():
    ids = torch.tensor([1, 2, 1, 3], device="cuda")
    d = torch.ones(4, 16, device="cuda")
    d[1, 3] = float("inf")
    d[3, 4] = float("nan")
    dw = torch.empty(5, 16, device="cuda")
    runner(5, 16, 4).wgrad(ids, d, dw)
    assert (dw[1] == 2).all() and dw[2, 3] == float("inf") and torch.isnan(dw[3, 4])
    assert torch.isfinite(dw[[0, 1, 4]]).all() and torch.isfinite(dw).sum() == 5 * 16 - 2


def test_no_tokens_and_shorter_batches():
    r = runner(20, 8, 5000)
    dw = torch.ones(20, 8, device="cuda")
    ids, d = torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, 8, device="cuda")
    r.wgrad(ids, d, dw, accumulate=True)
    assert (dw == 1).all()
    r.wgrad(ids, d, dw)
    assert (dw == 0).all()
    for n in (1, 9, 4736, 4737, 5000):
        ids = torch.arange(n, device="cuda") % 20
        r.wgrad(ids, torch.ones(n, 8, device="cuda"), dw)
        assert torch.equal(dw[:, 0], torch.bincount(ids, minlength=20).float())


def test_gradient_against_differences():
    """f = sum(w * out) is linear in the table: the gradient is its difference quotient for any step."""
    V, D, T = 6, 5, 11
    g = torch.Generator(device="cuda").manual_seed(0)
    table, w = torch.randn(V, D, generator=g, device="cuda"), torch.randn(T, D, generator=g, device="cuda")
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    r = runner(V, D, T, scale=2.0)
    dw, out = torch.empty(V, D, device="cuda"), torch.empty(T, D, device="cuda")
    r.wgrad(ids, w, dw)

    def f(t):
        r.forward(t, ids, out)
        return (out.double() * w.double()).sum()

    for v in range(V):
        for c in range(D):
            up, down = table.clone(), table.clone()
            up[v, c], down[v, c] = table[v, c] + 0.5, table[v, c] - 0.5
            want = (f(up) - f(down)) / (up[v, c].double() - down[v, c].double())
            # sums of T D terms of size up to about 2 * 4 * 4 in 64 bits; out is rounded once, at most 10 * 2^-24 a term
            assert abs(dw[v, c].double() - want) <= T * (10 * 4 + 8) * 2.0 ** -24


def test_same_bits_on_a_stream_and_in_a_graph():
    V, D, T = 9000, 256, 6000
    g = torch.Generator(device="cuda").manual_seed(3)
    ids, d = zipf(T, V, g), torch.randn(T, D, generator=g, device="cuda", dtype=torch.float32)
    r = runner(V, D, T)
    dw, other = torch.empty(V, D, device="cuda"), torch.empty(V, D, device="cuda")
    r.wgrad(ids, d, dw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r.wgrad(ids, d, other, stream=s)
    s.synchronize()
    assert torch.equal(dw, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.wgrad(ids, d, other)
    ids2 = zipf(T, V, g)
    r.wgrad(ids2, d, dw)
    ids.copy_(ids2)
    other.fill_(5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dw, other)


def test_runner_refuses_what_the_call_could_not_read():
    r = runner(10, 8, 6, bf16=True)
    ids, d, dw = torch.zeros(6, dtype=torch.int64, device="cuda"), torch.zeros(6, 8, device="cuda", dtype=BF), torch.zeros(10, 8, device="cuda")
    for args in ((ids.int(), d, dw), (ids.cpu(), d, dw), (torch.zeros(7, dtype=torch.int64, device="cuda"), d, dw),
                 (ids, d.float(), dw), (ids, d[:5], dw), (ids, d, dw[:9]), (ids, d, dw.double()), (ids[::2], d[:3], dw)):
        with pytest.raises(ValueError):
            r.wgrad(*args)
    for args in ((dw[:9], ids, d), (dw, ids, d.float()), (dw.double(), ids, d)):
        with pytest.raises(ValueError):
            r.forward(*args)
