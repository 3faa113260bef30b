"""Log probabilities of given tokens, entropy, top alternatives and their gradient against the definition in 64 bits.

Tolerances, in units u = 2^-24 (half a step of fp32).  A thread adds at most ceil(V / 256) terms in a row, then a tree of 5
shuffles, 8 warps and 8 CTAs: S is off by at most (V / 256 + 24) u relative to itself, plus the error of a term: exp2 of the
hardware 4 u, its argument a = d * c twice rounded (and c itself), 3 u |a| ln2; the weighted mean of |a| is at most
log2(V) + 2.  So rel(S) <= r = (V / 256 + 28 + 3 (log2 V + 2)) u.
  lse, logp:  r + 4 u (|lse| or |x_y - M| + |log S|) from the last products, sums and the logarithm
  entropy:    W / S is at most log2(V) + 2 in size and off by 2 r relative to that: r + 2 r ln2 (log2 V + 2) + 4 u (1 + log V)
  gradient:   p_j off by q_j = r + (4 + 3 |a_j|) u relative, the bracket by 8 u of its largest term, the rounding of the
              output half a step of its type, the given token's entry by u |alpha| scale more
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
IGN = -100


def half_step(dt):
    return torch.finfo(dt).eps / 2


def definition(x, y, scale, ignore=IGN):
    x = x.double() * scale
    M = x.amax(1, keepdim=True)
    d = torch.where(torch.isneginf(M), torch.full_like(x, -math.inf), x - M)
    e = torch.exp(d)
    S = e.sum(1, keepdim=True)
    lse = (M + torch.log(S))[:, 0]
    p = torch.where(S > 0, e / S, torch.zeros_like(e))
    lp = d - torch.log(S)
    H = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    given = (y >= 0) & (y < x.shape[1])
    logp = lp.gather(1, y.clamp(0, x.shape[1] - 1)[:, None])[:, 0]
    logp = torch.where(torch.isneginf(M[:, 0]), torch.full_like(logp, -math.inf), logp)
    logp = torch.where(given, logp, torch.full_like(logp, math.nan))
    logp = torch.where(y == ignore, torch.zeros_like(logp), logp)
    return dict(lse=lse, H=H, logp=logp, p=p, lp=lp, d=d, S=S[:, 0], M=M[:, 0], given=given)


def rel_S(V):
    return (V / 256 + 28 + 3 * (math.log2(max(V, 2)) + 2)) * U


def near(got, want, tol, what):
    got, want = got.double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    rest = ~fine & ~torch.isnan(want)
    assert torch.equal(got[rest], want[rest]), what
    tol = tol if isinstance(tol, torch.Tensor) else torch.full_like(want, tol)
    off = ((got - want).abs() - tol)[fine]
    assert off.numel() == 0 or off.max().item() <= 0, (what, off.max().item())


def check_stats(run, n, D, V):
    r = rel_S(V)
    logS = torch.log(D["S"]).abs().nan_to_num(0, 0, 0)
    near(run.lse[:n], D["lse"], r + 4 * U * (D["lse"].abs().nan_to_num(0, 0, 0) + logS), "lse")
    near(run.logp[:n], D["logp"], r + 4 * U * (D["logp"].abs().nan_to_num(0, 0, 0) + 2 * logS), "logp")
    near(run.entropy[:n], D["H"], r + 2 * r * math.log(2) * (math.log2(V) + 2) + 4 * U * (1 + math.log(V)), "entropy")


def check_grad(got, D, y, V, scale, alpha, beta, dt, from_lse=False, ignore=IGN):
    p, lp, H = D["p"], D["lp"], D["H"][:, None]
    alpha, beta = alpha.double()[:, None], (beta if beta is not None else torch.zeros_like(alpha)).double()[:, None]
    hot = torch.zeros_like(p)
    hot.scatter_(1, y.clamp(0, V - 1)[:, None], 1.0)
    lpz = torch.where(p > 0, lp, torch.zeros_like(lp))
    want = scale * (alpha * (hot - p) - beta * torch.where(p > 0, p * (lpz + H), torch.zeros_like(p)))
    want = torch.where(torch.isneginf(D["M"])[:, None], torch.zeros_like(want), want)
    want = torch.where(D["given"][:, None], want, torch.full_like(want, math.nan))
    want = torch.where((y == ignore)[:, None], torch.zeros_like(want), want)
    a = (D["d"] / math.log(2)).clamp(min=-150).nan_to_num(0, 0, 0)
    q = rel_S(V) + (4 + 3 * a.abs()) * U
    if from_lse:            # p = exp(x - lse) with lse rounded to fp32 and off by its own tolerance; not from |lse| = 4096 on
        big = (D["lse"].abs()[:, None] + (D["d"] + D["M"][:, None]).abs()).nan_to_num(0, 0, 0)
        q = q + torch.where(D["lse"].abs()[:, None] < 4096, 6 * U * big.clamp(max=1e5), torch.zeros_like(big)) + rel_S(V)
    # the bracket's largest terms, and the entropy that the kernel uses being off by its own tolerance
    eH = rel_S(V) * (1 + 2 * math.log(2) * (math.log2(max(V, 2)) + 2)) + 4 * U * (1 + math.log(V))
    size = alpha.abs() + beta.abs() * (H.abs() + lpz.abs() + 2 * torch.log(D["S"]).abs()[:, None].nan_to_num(0, 0, 0))
    tol = scale * p * (size * (q + 8 * U) + beta.abs() * eH) + 2 * U * scale * alpha.abs() * hot
    # products below the smallest normal number are flushed
    near(got, want, half_step(dt) * want.abs().nan_to_num(0) * (1 + 2.0 ** -7) + tol.nan_to_num(0) + 2.0 ** -120, "gradient")


def top_of(x, k):
    v, i = torch.sort(x.double(), dim=1, descending=True, stable=True)
    return v[:, :k], i[:, :k]


def make(T, V, dt, pad=0, off=0, seed=0, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.zeros(off + T * (V + pad) + 16, device="cuda", dtype=dt)
    body = flat[off:off + T * (V + pad)].view(T, V + pad)
    body.copy_(torch.randn(T, V + pad, generator=g, device="cuda") * spread)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    return body[:, :V], y, body


def runner(T, V, dt, **kw):
    from paper_2505_05086_b200.runner import LogprobRunner
    return LogprobRunner(T, V, bf16=dt == torch.bfloat16, **kw)


SIZES = [(1, 1, 0, 0), (3, 2, 1, 1), (2, 7, 0, 3), (5, 33, 2, 0), (4, 257, 0, 1), (7, 1000, 24, 0), (150, 513, 0, 5),
         (2, 32000, 0, 0), (300, 32000, 8, 1), (3, 50257, 0, 0), (2, 131073, 7, 1), (1, 400003, 0, 0), (2, 950001, 1, 0),
         # many rows, from where small CTAs take them, on both sides of their lines (granules of 8 or 4 values)
         (600, 1, 0, 1), (600, 300, 1, 3), (593, 641, 0, 1), (593, 1275, 2, 0), (600, 2041, 0, 1), (592, 4089, 0, 5),
         (600, 8401, 0, 0), (592, 16795, 0, 2)]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,pad,off", SIZES)
def test_forward_and_gradients_match_the_definition(T, V, pad, off, dt):
    x, y, _ = make(T, V, dt, pad, off, seed=V + T)
    if T > 2:
        y[1] = IGN
    k, scale = min(20, V), 0.75
    run = runner(T, V, dt, scale=scale, top_k=k)
    run.forward(x, y)
    D = definition(x, y, scale)
    check_stats(run, T, D, V)
    v, i = top_of(x, k)
    assert torch.equal(run.top_ids, i)
    want = v * scale - D["lse"][:, None]
    near(run.top_logp, want, rel_S(V) + 6 * U * (want.abs() + torch.log(D["S"])[:, None].abs()), "top_logp")
    g = torch.Generator(device="cuda").manual_seed(1)
    alpha, beta = torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
    for b in (None, beta):
        for form in ("backward", "loss"):
            whole = torch.full((T, V + pad + 3), 7.0, device="cuda", dtype=dt)
            getattr(run, form)(x, y, alpha, b, whole[:, :V])
            check_grad(whole[:, :V], D, y, V, scale, alpha, b, dt, from_lse=form == "backward")
            assert (whole[:, V:] == 7).all()                       # between vocab and ld_grad: as it was
    check_stats(run, T, D, V)                                       # as loss() left them


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,times", [(5, 1), (600, 1), (40000, 1), (150000, 1), (5, 70), (300, 70), (1600, 70), (6000, 70)])
def test_masked_entries_and_rows_without_any(V, times, dt):
    T = 9
    x, y, _ = make(T, V, dt, seed=3)
    lowest = torch.finfo(dt).min
    x[0, : V // 2] = -math.inf
    y[0] = V - 1
    x[1] = -math.inf                                               # nothing left
    x[2] = lowest                                                  # all equal, at the type's lowest value
    x[3, 1:] = -math.inf                                           # one left
    y[3] = 0
    x[4, 1:] = lowest
    y[4] = 0
    x[5], y[5] = -math.inf, IGN
    y[6] = IGN
    x[7, 0], y[7] = -math.inf, 0                                   # the given token is masked
    x[8] = 2.5                                                     # all equal
    x, y = x.repeat(times, 1), y.repeat(times)
    T *= times
    k = min(32, V)
    run = runner(T, V, dt, top_k=k)
    run.forward(x, y)
    D = definition(x, y, 1.0)
    check_stats(run, T, D, V)
    v, i = top_of(x, k)
    assert torch.equal(run.top_ids, i)
    dead = torch.isneginf(D["M"])
    assert torch.isneginf(run.top_logp[dead]).all()
    # from the maximum: next to the type's lowest value even 64 bits lose log V in x - lse
    want = (v - D["M"][:, None] - torch.log(D["S"])[:, None])[~dead]
    near(run.top_logp[~dead], want, rel_S(V) + 6 * U * (want.abs() + math.log(V) + 1).nan_to_num(0, 0, 0), "top_logp")
    alpha, beta = torch.linspace(0.5, 2, T, device="cuda"), torch.linspace(-1, 1, T, device="cuda")
    for form in ("backward", "loss"):
        out = torch.empty(T, V, device="cuda", dtype=dt)
        getattr(run, form)(x, y, alpha, beta, out)
        keep = torch.tensor([t % 9 != 7 for t in range(T)], device="cuda")   # log p of the masked token: -inf * 0 by the formula
        sub = {n: q[keep] for n, q in D.items()}
        check_grad(out[keep], sub, y[keep], V, 1.0, alpha[keep], beta[keep], dt, from_lse=form == "backward")
        assert torch.isfinite(out).all()
        for t in (1, 5, 6):
            assert (out[t::9] == 0).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [70, 50000])
@pytest.mark.parametrize("level", [1000.0, -5000.0, 1e6, -1e30])
def test_logits_far_from_zero(level, V, dt):
    """All logits of some rows at a level where lse in fp32 says little about their differences."""
    T = 5
    x, y, _ = make(T, V, torch.float32, seed=11)
    x[1:4] = (x[1:4] * abs(level) * 2.0 ** -7 + level) if abs(level) < 1e5 else level
    x = x.to(dt)
    y[3] = IGN
    run = runner(T, V, dt)
    run.forward(x, y)
    D = definition(x, y, 1.0)
    check_stats(run, T, D, V)
    alpha, beta = torch.linspace(0.5, 2, T, device="cuda"), torch.linspace(-1, 1, T, device="cuda")
    for form in ("backward", "loss"):
        out = torch.empty(T, V, device="cuda", dtype=dt)
        getattr(run, form)(x, y, alpha, beta, out)
        check_grad(out, D, y, V, 1.0, alpha, beta, dt, from_lse=form == "backward")
        again = x.clone()
        getattr(run, form)(again, y, alpha, beta, again)
        assert torch.equal(again, out)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,times", [(6, 1), (40000, 1), (6, 100), (1700, 100), (9000, 100)])
def test_nan_inf_and_targets_outside_the_vocabulary(V, times, dt):
    T = 6
    x, y, _ = make(T, V, dt, seed=4)
    x[0, V - 1] = math.nan
    x[1, 0] = math.inf
    x[2, 1], y[2] = math.nan, IGN
    y[3], y[4] = V, -7
    x[5] = math.nan
    x, y = x.repeat(times, 1), y.repeat(times)
    T *= times
    run = runner(T, V, dt, top_k=4)
    run.forward(x, y)
    out = torch.empty(T, V, device="cuda", dtype=dt)
    one = torch.ones(T, device="cuda")

    def rows(*which):
        return torch.tensor([t % 6 in which for t in range(T)], device="cuda")

    def look():
        for o in (run.lse, run.entropy):
            assert torch.isnan(o[rows(0, 1, 2, 5)]).all() and torch.isfinite(o[rows(3, 4)]).all()
        assert torch.isnan(run.logp[rows(0, 1, 3, 4, 5)]).all() and (run.logp[rows(2)] == 0).all()

    look()
    assert torch.isnan(run.top_logp[rows(0, 1, 2, 5)]).all()
    assert (run.top_ids[rows(0, 1, 2, 5)] == torch.arange(4, device="cuda")).all()
    assert torch.equal(run.top_ids[rows(3, 4)], top_of(x[rows(3, 4)], 4)[1])
    for form in ("backward", "loss"):
        out.fill_(3)
        getattr(run, form)(x, y, one, one, out)
        assert torch.isnan(out[rows(0, 1, 3, 4, 5)]).all() and (out[rows(2)] == 0).all()
    look()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_ties_go_to_the_lowest_index(dt):
    """Many equal values: more candidates than the kernel's list holds, in one CTA and over a cluster."""
    for T, V in ((200, 9000), (1, 60000), (600, 1000), (600, 4000)):
        g = torch.Generator(device="cuda").manual_seed(5)
        x = torch.randint(-2, 3, (T, V), generator=g, device="cuda").to(dt)
        x[0, 17] = -0.0
        run = runner(T, V, dt, top_k=32)
        run.forward(x, torch.zeros(T, dtype=torch.int64, device="cuda"))
        assert torch.equal(run.top_ids, top_of(x + 0.0, 32)[1])
        z = torch.zeros(T, V, device="cuda", dtype=dt)
        run.forward(z, torch.zeros(T, dtype=torch.int64, device="cuda"))
        assert torch.equal(run.top_ids, torch.arange(32, device="cuda").expand(T, 32))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", ["loss", "backward"])
@pytest.mark.parametrize("T,V,off", [(3, 50257, 1), (170, 1003, 0), (1, 900001, 3)])
def test_gradient_in_place(T, V, off, dt, form):
    x, y, _ = make(T, V, dt, 0, off, seed=6)
    alpha, beta = torch.randn(T, device="cuda"), torch.randn(T, device="cuda")
    run = runner(T, V, dt)
    run.forward(x, y)
    other = torch.empty(T, V, device="cuda", dtype=dt)
    getattr(run, form)(x, y, alpha, beta, other)
    getattr(run, form)(x, y, alpha, beta, x)
    assert torch.equal(x, other)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", ["loss", "backward"])
@pytest.mark.parametrize("T,V,gap", [(3, 50257, 0), (700, 1003, 1), (700, 8, 5)])
def test_gradient_between_the_rows_of_the_logits(T, V, gap, dt, form):
    x, y, _ = make(T, V, dt, 0, 0, seed=8)
    alpha, beta = torch.randn(T, device="cuda"), torch.randn(T, device="cuda")
    run = runner(T, V, dt)
    both = torch.full((T, 2 * V + gap), 7.0, device="cuda", dtype=dt)
    both[:, :V] = x
    run.forward(both[:, :V], y)
    other = torch.empty(T, 2 * V + gap, device="cuda", dtype=dt)
    apart = other[:, V:2 * V]
    getattr(run, form)(both[:, :V], y, alpha, beta, apart)
    getattr(run, form)(both[:, :V], y, alpha, beta, both[:, V:2 * V])
    assert torch.equal(both[:, V:2 * V], apart)
    assert torch.equal(both[:, :V], x) and (both[:, 2 * V:] == 7).all()


def test_gradient_against_differences():
    T, V, h = 4, 40, 0.02
    x, y, _ = make(T, V, torch.float32, seed=7, spread=1.0)
    a, b = torch.randn(T, device="cuda", dtype=torch.float64), torch.randn(T, device="cuda", dtype=torch.float64)
    run = runner(T, V, torch.float32, scale=1.5)
    out = torch.empty_like(x)
    run.loss(x, y, a.float(), b.float(), out)

    def f(z):
        D = definition(z, y, 1.5)
        return a.float().double() * D["logp"] + b.float().double() * D["H"]

    # central differences of the definition are off by h^2 / 6 times a third derivative: at most about
    # (1.5^3)(|a| + 4 |b| (1 + log V)) in size here
    tol = h * h / 6 * 1.5 ** 3 * 8 * (a.abs() + 4 * b.abs() * (1 + math.log(V)))
    for j in range(V):
        e = torch.zeros(V, device="cuda", dtype=torch.float64)
        e[j] = h
        want = (f(x.double() + e) - f(x.double() - e)) / (2 * h)
        assert ((out[:, j].double() - want).abs() <= tol).all()


def test_shorter_batches_leave_the_other_rows():
    run = runner(6, 100, torch.float32, top_k=3)
    for o in (run.logp, run.lse, run.entropy, run.top_logp):
        o.fill_(9)
    x, y, _ = make(4, 100, torch.float32)
    run.forward(x, y)
    for o in (run.logp, run.lse, run.entropy, run.top_logp):
        assert (o[4:] == 9).all() and not (o[:4] == 9).any()
    run.forward(x[:0], y[:0])                                       # nothing to do


def test_same_bits_again_on_a_stream_and_in_a_graph():
    T, V = 33, 50257
    x, y, _ = make(T, V, torch.bfloat16, seed=8)
    run = runner(T, V, torch.bfloat16, top_k=8)
    alpha, out = torch.randn(T, device="cuda"), torch.empty(T, V, device="cuda", dtype=torch.bfloat16)

    def both():
        run.forward(x, y)
        run.loss(x, y, alpha, alpha, out)
        return [t.clone() for t in (run.logp, run.entropy, run.lse, run.top_logp, run.top_ids, out)]

    first = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = both()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run.forward(x, y)
        run.loss(x, y, alpha, alpha, out)
    x2, y2, _ = make(T, V, torch.bfloat16, seed=9)
    keep = x.clone(), y.clone()
    x.copy_(x2), y.copy_(y2)
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (run.logp, run.entropy, run.lse, run.top_logp, run.top_ids, out)]
    assert all(torch.equal(a, b) for a, b in zip(got, both()))
    x.copy_(keep[0]), y.copy_(keep[1])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, [run.logp, run.entropy, run.lse, run.top_logp, run.top_ids, out]))


def test_runner_refuses_what_the_call_could_not_read():
    run = runner(4, 50, torch.bfloat16, top_k=2)
    x, y, body = make(4, 50, torch.bfloat16, pad=2)
    out, a = torch.empty(4, 50, device="cuda", dtype=torch.bfloat16), torch.ones(4, device="cuda")
    for bad in (x.float(), x[:, :49], x.t(), x.cpu(), torch.cat([x, x])):
        with pytest.raises(ValueError):
            run.forward(bad, y)
    for bad in (y.int(), y[:3], y.cpu(), y.repeat(2)[::2]):
        with pytest.raises(ValueError):
            run.forward(x, bad)
    for bad in (a.double(), a[:2], a.cpu()):
        with pytest.raises(ValueError):
            run.loss(x, y, bad, None, out)
        with pytest.raises(ValueError):
            run.backward(x, y, a, bad, out)
    from paper_2505_05086_b200 import AsiError
    with pytest.raises(AsiError):                                   # over the logits, but not row for row
        run.loss(x, y, a, None, body.view(-1)[1:1 + 4 * 50].view(4, 50))


def test_results_that_are_not_asked_for():
    """Through the binding: no entropy, no alternatives."""
    from paper_2505_05086_b200 import binding as B
    T, V = 5, 700
    x, y, _ = make(T, V, torch.float32, seed=12)
    ref = runner(T, V, torch.float32)
    ref.forward(x, y)
    d = B.LogprobDesc(0, 0, T, V, V, V, IGN, 1.0)
    s = torch.cuda.current_stream().cuda_stream
    logp, lse, out, want = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    B.token_logprobs(d, x.data_ptr(), y.data_ptr(), logp.data_ptr(), 0, lse.data_ptr(), stream=s)
    assert torch.equal(logp, ref.logp) and torch.equal(lse, ref.lse)
    one = torch.ones(T, device="cuda")
    logp.fill_(0)
    B.token_loss(d, x.data_ptr(), y.data_ptr(), one.data_ptr(), 0, logp.data_ptr(), 0, lse.data_ptr(), out.data_ptr(), s)
    ref.loss(x, y, one, None, want)
    assert torch.equal(logp, ref.logp) and torch.equal(out, want)
    B.token_logprobs_grad(d, x.data_ptr(), y.data_ptr(), lse.data_ptr(), 0, one.data_ptr(), 0, out.data_ptr(), s)
    ref.backward(x, y, one, None, want)
    assert torch.equal(out, want)
