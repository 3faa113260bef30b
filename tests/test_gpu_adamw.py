"""AdamW over many tensors.  m and v are separately rounded fp32 operations, so states (and the 8-bit codes and scales of m)
have to equal a restatement in numpy's fp32 bit for bit; sqrt(v) is the hardware's, off by at most 2^-23 of its value, so its
codes and scales have to be those of a value within that.  The weight, u = 2^-24 a rounding: the root 2 u, its constant, the
constant eps, the denominator, the step's constant and two products u each, the reciprocal 2 u, so 10 u |update| at most,
where m and v are taken as rounded; 2 u |w| for the decay and its product; then half a step of the weight's type."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.02)
U = 2.0 ** -24


def decode(codes, scales):
    e = scales.view(torch.uint8).cpu().numpy().astype(np.int64) - 127
    c = codes.view(torch.float8_e4m3fn).float().cpu().numpy()
    return (c * np.exp2(e.astype(np.float32))[np.arange(len(c)) // 256].astype(np.float32)).astype(np.float32)


def encode(x, sqrt_of_v):
    """codes and scale bytes of a flat fp32 array, from their definition"""
    n = len(x)
    b = np.zeros(-(-n // 256) * 256, np.float32)
    b[:n] = x
    b = b.reshape(-1, 256)
    a = np.where(np.isfinite(b), np.abs(b), 0).max(1).astype(np.float64)
    k = np.zeros(len(a), np.int64)
    for i, t in enumerate(a):
        if t > 0:
            k[i] = max(math.frexp(t)[1] - 9 + (math.frexp(t)[0] > 0.875), -126)
    with np.errstate(invalid="ignore"):
        q = (b * np.exp2(-k.astype(np.float64))[:, None]).astype(np.float32)
    q = np.where(np.isinf(q), np.nan, q)
    c = torch.from_numpy(q).to(torch.float8_e4m3fn)
    if sqrt_of_v:
        f = c.float().numpy()
        c = torch.from_numpy(np.where((b > 0) & (f == 0), np.float32(2.0 ** -9), f)).to(torch.float8_e4m3fn)
    return c.view(-1)[:n], (k + 127).astype(np.uint8)


def restate(w, g, m, v, t, h, gs=None, lr=None, r=None):
    """One step on flat numpy arrays: fp32 states as the kernel rounds them, the weight in 64 bits."""
    f = np.float32
    g = g.astype(f)
    if gs is not None:
        g = (g * f(gs)).astype(f)
    with np.errstate(over="ignore", invalid="ignore"):
        m = (m * f(h["beta1"])).astype(f) + (g * f(1 - h["beta1"])).astype(f)
        v = (v * f(h["beta2"])).astype(f) + ((g * g).astype(f) * f(1 - h["beta2"])).astype(f)
        r = np.sqrt(v)
        lr = h["lr"] if lr is None else lr
        up = lr / (1 - h["beta1"] ** t) * m.astype(np.float64) / (r.astype(np.float64) / math.sqrt(1 - h["beta2"] ** t) + h["eps"])
        new = w.astype(np.float64) * (1 - lr * h["weight_decay"]) - up
    return new, m, v, r, up


def build(sizes, wt, gt, bits8, copy=False, off=0, seed=0):
    from paper_2505_05086_b200.runner import AdamWRunner
    g = torch.Generator(device="cuda").manual_seed(seed)

    def some(dt, n, scale):
        x = torch.zeros(n + off + 16, device="cuda", dtype=dt)[off:off + n]
        x.copy_(torch.randn(n, generator=g, device="cuda") * scale)
        return x
    ws = [some(wt, n, 0.05) for n in sizes]
    gs = [some(gt, n, 1e-3 * 10 ** (i % 4)) for i, n in enumerate(sizes)]
    cs = [some(BF, n, 1.0) for n in sizes] if copy else None
    return AdamWRunner(ws, gs, bits8=bits8, copies=cs)


def states_np(r, i):
    if r.bits8:
        m = decode(r.exp_avg[i], r.exp_avg_scale[i])
        s = decode(r.exp_avg_sq[i], r.exp_avg_sq_scale[i])
        return m, (s * s).astype(np.float32)
    return r.exp_avg[i].cpu().numpy(), r.exp_avg_sq[i].cpu().numpy()


def check_step(r, t, h=HYPER, gs=None, lr=None, slack=0.0, call=None, **kw):
    before = [(w.float().cpu().numpy().ravel(), g.float().cpu().numpy().ravel(), *states_np(r, i))
              for i, (w, g) in enumerate(zip(r.weights, r.grads))]
    (call or r.step)(**{**h, **kw})
    torch.cuda.synchronize()
    for i, (w, g, m, v) in enumerate(before):
        new, m, v, rt, up = restate(w, g, m, v, t, h, gs, lr)
        got = r.weights[i].double().cpu().numpy().ravel()
        wt = r.weights[i].dtype
        tol = U * (2 * np.abs(w) + (10 + slack) * np.abs(up)) + torch.finfo(wt).eps / 2 * np.abs(new) + 2.0 ** -140
        assert (np.abs(got - new) <= tol).all(), (i, np.max(np.abs(got - new) / tol))
        if r.copies[i] is not None:
            # rounded from the fp32 value, not from the stored one
            tol = U * (2 * np.abs(w) + (10 + slack) * np.abs(up)) + torch.finfo(BF).eps / 2 * np.abs(new) * (1 + 2.0 ** -7) + 2.0 ** -140
            assert (np.abs(r.copies[i].double().cpu().numpy() - new) <= tol).all()
        if r.bits8:
            c, e = encode(m, False)
            assert np.array_equal(r.exp_avg_scale[i].view(torch.uint8).cpu().numpy(), e), i
            assert torch.equal(r.exp_avg[i].view(torch.uint8).cpu(), c.view(torch.uint8)), i
            got_e = r.exp_avg_sq_scale[i].view(torch.uint8).cpu().numpy()
            (_, e0), (_, e1) = (encode((rt.astype(np.float64) * (1 + s * 2.0 ** -23)).astype(np.float32), True) for s in (-1, 1))
            assert ((got_e >= e0) & (got_e <= e1)).all(), i
            # codes of values at either end of the root's error, under the scales that are there
            got = r.exp_avg_sq[i].float().cpu().numpy()
            lo, hi = ((rt.astype(np.float64) * (1 + s * 2.0 ** -23) / np.exp2(got_e.astype(np.float64) - 127)[np.arange(len(rt)) // 256])
                      for s in (-1, 1))
            lo, hi = (torch.from_numpy(np.minimum(x, 448).astype(np.float32)).to(torch.float8_e4m3fn).float().numpy() for x in (lo, hi))
            lo, hi = (np.where((rt > 0) & (x == 0), np.float32(2.0 ** -9), x) for x in (lo, hi))
            assert ((got >= lo) & (got <= hi)).all(), i
        else:
            assert np.array_equal(r.exp_avg[i].cpu().numpy(), m) and np.array_equal(r.exp_avg_sq[i].cpu().numpy(), v), i


SIZES = [1, 2, 7, 8, 255, 256, 257, 1000, 4096, 4097, 20000, 0, 3]


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("wt,gt", [(F32, F32), (F32, BF), (BF, F32), (BF, BF)])
@pytest.mark.parametrize("off", [0, 1, 4])
def test_steps_match_a_restatement(wt, gt, bits8, off):
    r = build(SIZES, wt, gt, bits8, copy=wt == F32, off=off)
    for t in (1, 2, 3):
        check_step(r, t)


def test_more_tensors_than_one_launch_holds():
    sizes = [1 + (37 * i) % 900 for i in range(1000)]
    check_step(build(sizes, F32, F32, True), 1)


def test_a_large_tensor():
    r = build([3_000_001], F32, BF, True, copy=True)
    check_step(r, 1)
    check_step(r, 2)


@pytest.mark.parametrize("bits8", [False, True])
def test_extreme_gradients(bits8):
    """Zeros, subnormal and huge values in one block: nothing is lost that would let a step explode."""
    r = build([512, 300], F32, F32, bits8)
    g = r.grads[0]
    g.zero_()
    g[3], g[5], g[7], g[9] = 1e-30, 3e4, -2e-7, 1e-41
    r.grads[1].zero_()
    for t in (1, 2, 3):
        check_step(r, t)
    # an element far below the block's largest keeps a denominator: no step larger than the bounded ratio m / sqrt(v) allows
    w = r.weights[0].clone()
    for t in range(4, 12):
        r.step(**HYPER)
    assert torch.isfinite(r.weights[0]).all() and (r.weights[0] - w).abs().max() < 8 * 20 * HYPER["lr"]


def test_values_that_are_not_finite_stay_with_their_elements():
    for bits8 in (False, True):
        r = build([600], F32, F32, bits8)
        r.grads[0][5], r.grads[0][300], r.grads[0][301] = math.nan, math.inf, -math.inf
        ref = build([600], F32, F32, bits8)
        ref.grads[0][5] = ref.grads[0][300] = ref.grads[0][301] = 0.0
        r.step(**HYPER), ref.step(**HYPER)
        bad = torch.zeros(600, dtype=torch.bool, device="cuda")
        bad[[5, 300, 301]] = True
        assert torch.equal(r.weights[0][~bad], ref.weights[0][~bad])
        assert torch.equal(r.exp_avg[0].float()[~bad], ref.exp_avg[0].float()[~bad])
        assert torch.isnan(r.weights[0][bad]).all()
        if bits8:
            assert torch.isnan(r.exp_avg[0].float()[bad]).all() and torch.isnan(r.exp_avg_sq[0].float()[bad]).all()


@pytest.mark.parametrize("bits8", [False, True])
def test_gradient_scale_learning_rate_and_step_on_the_device(bits8):
    r = build([5000, 33], F32, BF, bits8)
    gs, lr = torch.tensor([0.37], device="cuda"), torch.tensor(2e-3, device="cuda")
    step = torch.tensor([1], dtype=torch.int64, device="cuda")
    # 1 - beta^t from fp32 logarithms and expm1: 8 u relative on each correction more
    check_step(r, 1, gs=np.float32(0.37), lr=float(lr), lr_dev=None, slack=24, call=lambda lr_dev=None, **h: r.step(**{**h, "lr": lr, "step": step, "grad_scale": gs}))
    step.fill_(900)
    check_step(r, 900, gs=np.float32(0.37), lr=float(lr), lr_dev=None, slack=24, call=lambda lr_dev=None, **h: r.step(**{**h, "lr": lr, "step": step, "grad_scale": gs}))
    check_step(r, 901, lr=float(lr), lr_dev=None, slack=8, call=lambda lr_dev=None, **h: r.step(**{**h, "lr": lr, "step": 901}))
    step.fill_(902)
    check_step(r, 902, slack=24, call=lambda **h: r.step(**{**h, "step": step}))


@pytest.mark.parametrize("bits8", [False, True])
def test_a_captured_step_reads_step_and_rate_when_replayed(bits8):
    a, b = (build([4000, 77, 9], F32, F32, bits8, seed=2) for _ in range(2))
    step, lr = torch.tensor([1], dtype=torch.int64, device="cuda"), torch.tensor([1e-3], device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(lr=lr, step=step)
        step += 1
    for t in range(1, 6):
        lr.fill_(1e-3 / t)
        graph.replay()
        b.step(lr=lr, step=torch.tensor([t], dtype=torch.int64, device="cuda"))
    torch.cuda.synchronize()
    for x, y in zip(a.weights + a.exp_avg + a.exp_avg_sq, b.weights + b.exp_avg + b.exp_avg_sq):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert int(step) == 6


def test_states_can_be_carried_to_another_runner():
    from paper_2505_05086_b200.runner import AdamWRunner
    a = build([700, 20], F32, F32, True, seed=4)
    a.step(**HYPER)
    b = AdamWRunner([w.clone() for w in a.weights], a.grads, bits8=True, exp_avg=[x.clone() for x in a.exp_avg],
                    exp_avg_sq=[x.clone() for x in a.exp_avg_sq], exp_avg_scale=[x.clone() for x in a.exp_avg_scale],
                    exp_avg_sq_scale=[x.clone().view(torch.uint8) for x in a.exp_avg_sq_scale])
    a.step(**HYPER), b.step(step=2, **HYPER)
    assert all(torch.equal(x, y) for x, y in zip(a.weights, b.weights)) and a.t == b.t == 2


def test_runner_refuses_what_the_call_could_not_read():
    from paper_2505_05086_b200 import AsiError
    from paper_2505_05086_b200.runner import AdamWRunner
    w, g = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    for ws, gs, kw in (([], [], {}), ([w], [], {}), ([w], [g[:63]], {}), ([w.half()], [g], {}), ([w], [g.double()], {}),
                       ([w[::2]], [g[:32]], {}), ([w], [g], dict(copies=[w])), ([w], [g], dict(exp_avg=[w[:3]])),
                       ([w, w.bfloat16()], [g, g], {}), ([w], [g.cpu()], {}), ([w.cpu()], [g], {})):
        with pytest.raises(ValueError):
            AdamWRunner(ws, gs, **kw)
    with pytest.raises(AsiError):                                   # the same weight twice
        AdamWRunner([w, w], [g, g]).step()
    r = AdamWRunner([w], [g])
    for kw in (dict(lr=-1.0), dict(beta1=1.0), dict(eps=0.0), dict(step=0), dict(weight_decay=-0.1)):
        with pytest.raises(AsiError):
            r.step(**kw)
    with pytest.raises(ValueError):
        r.step(lr=torch.tensor(0.1))
