"""What the output layer's gradients are held to beyond their elementwise bounds, each by a quantity of its own."""
import pytest
import torch

from tests.block_util import U16, U32, head
from tests.test_gpu_head import DT, World

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


def far_world(T, V, offset, bf16, bf16_dw, **kw):
    """Logits around offset[0] * offset[1] whose products and sums are exact in fp32 (multiples of 1/8), and columns of x that are 1 in one row alone and
    meet zeros of w, so that dw holds G as it is."""
    w = World(T, V, 16 + T, bf16, bf16_dw, ignored=0.0, **kw)
    g = torch.Generator(device="cuda").manual_seed(V)
    x, t = torch.zeros(T, 16 + T, device="cuda"), torch.arange(T, device="cuda")
    x[:, 1:16] = torch.randint(-4, 5, (T, 15), generator=g, device="cuda").float()
    x[:, 0], x[t, 16 + t] = offset[0], 1.0
    k = torch.zeros(V, 16 + T, device="cuda")
    k[:, 1:16] = torch.randint(-2, 3, (V, 15), generator=g, device="cuda").float() / 8
    k[:, 0] = offset[1]
    w.x, w.w = x.to(DT[bf16]), k.to(DT[bf16])
    w.dlogp.fill_(0.75)
    return w


def check_far(w, gw):
    """G, as dw holds it, where lse is large: with |log p| <= 16 exponents are off by 2^-24 of |log p| and of the logit's distance from the maximum, twice at
    most, each times ln 2, the factor in them by as much, the power and the sum by 2^-21 together, and G's own rounding comes on top."""
    r = head(w.x, w.w, w.y, 1.0, -100, w.dlogp)
    got, want = gw[:, 16:].T.double(), r["G"]
    lp = r["p"].log()
    bound = 0.75 * r["p"] * ((8 * lp.abs() + 32) * U32) + (2 * U16 if w.bf16_dw else 4 * U32) * want.abs()
    assert (((got - want).abs() <= bound) | (lp < -16)).all()


@pytest.mark.parametrize("bf16,bf16_dw,offset", [(False, False, (64, 16)), (True, False, (64, 16)), (True, False, (-64, 16)), (True, True, (512, 256)),
                                                 (True, True, (-512, 256))])
@pytest.mark.parametrize("T,V", [(20, 600), (300, 1100)])
@pytest.mark.parametrize("chunk", [0, 512])
def test_gradient_of_large_logits(T, V, bf16, bf16_dw, offset, chunk):
    w = far_world(T, V, offset, bf16, bf16_dw, vocab_chunk=chunk)
    check_far(w, w.loss()["dw"])


@pytest.mark.parametrize("bf16,bf16_dw,offset", [(False, False, (64, 16)), (True, False, (64, 16)), (True, False, (-64, 16)), (True, True, (512, 256))])
@pytest.mark.parametrize("T,V", [(20, 600), (300, 1100)])
def test_gradient_apart_from_its_forward_pass_where_lse_is_large(T, V, bf16, bf16_dw, offset):
    """By an lse of 1024 that is rounded to fp32 p would be off by 2^-14 (half a step; 2^-7 at 131072), in all of a row alike."""
    w = far_world(T, V, offset, bf16, bf16_dw)
    gw = torch.empty(V, 16 + T, device="cuda", dtype=DT[bf16_dw])
    w.op.forward(w.x, w.w, w.y)
    lse = w.op.lse.clone()
    w.op.backward(w.x, w.w, w.y, w.dlogp, None, None, gw)
    check_far(w, gw)
    assert torch.equal(w.op.lse, lse)


def test_rows_near_and_far_in_one_call():
    """A row with a large lse changes nothing in the rows beside it."""
    near, far = far_world(40, 700, (4, 2), False, False), far_world(40, 700, (4, 2), False, False)
    far.x[::3, 0] = 512
    out = []
    for w in (near, far):
        gx, gw = torch.empty_like(w.x), torch.empty(700, 56, device="cuda")
        w.op.forward(w.x, w.w, w.y)
        w.op.backward(w.x, w.w, w.y, w.dlogp, None, gx, gw)
        out.append((gx, gw))
    keep = [t for t in range(40) if t % 3]
    assert torch.equal(out[0][0][keep], out[1][0][keep])
    assert torch.equal(out[0][1][:, [16 + t for t in keep]], out[1][1][:, [16 + t for t in keep]])


def test_a_bf16_dw_of_very_many_rows_is_not_biased():
    """Sums that stay in the tensor cores' accumulators are truncated at each step of 16 k: by 2^-24 of the sum so far, half an ulp, in the mean or more, always
    towards zero; 2^18 rows are 16384 steps, 5e-4 of the sum at least.  Rounding has no sign: the mean relative error of 255 x 64 values that lie anywhere
    in their binades (columns of x differ by up to 2), each rounded by 2^-8 / sqrt 3 at most in the mean square, is within 1.8e-5, and roundings of G (one
    value's are shared by 64 of dw, 2^18 of them average down by 512) add 4.4e-6 / 16 to that.  Three of these."""
    T, V, D = 1 << 18, 256, 64
    w = World(T, V, D, bf16=True, bf16_dw=True, ignored=0.0)
    column = 1 + torch.arange(D, device="cuda") / D
    w.x = ((1 + 0.25 * torch.rand(T, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))) * column).bfloat16()
    w.w = (w.w / column).bfloat16()
    w.y.fill_(0)
    w.dlogp.fill_(-1.0 / T)
    gw = torch.empty(V, D, device="cuda", dtype=torch.bfloat16)
    w.op.loss(w.x, w.w, w.y, w.dlogp, None, None, gw)
    want = torch.zeros(V, D, device="cuda", dtype=torch.float64)
    for t in range(0, T, 1 << 14):
        s = slice(t, t + (1 << 14))
        want += head(w.x[s], w.w, w.y[s], 1.0, -100, w.dlogp[s])["dw"]
    off = ((gw.double() - want) / want)[1:]
    assert abs(float(off.mean())) <= 5.4e-5


@pytest.mark.parametrize("T,V,D", [(1, 700, 64), (9, 9000, 264), (40, 1100, 75), (256, 2000, 136), (256, 600, 1032)])
@pytest.mark.parametrize("add", [False, True])
def test_a_bf16_dw_of_few_rows_is_rounded_once(T, V, D, add):
    """World.check's bounds of dw, but for G's rounding: two terms of bf16 leave 2^-17 of each entry (2^-8 twice, and what is left has the sign and half of the
    last step), and dw itself half a step."""
    w = World(T, V, D, bf16=True, bf16_dw=True, ignored=0.0 if T < 9 else 0.15)
    start = (torch.randn(V, D, device="cuda") / (4 * T)).bfloat16() if add else None
    got, r = w.loss(accumulate=add, start=start, dx=add), w.reference()      # (dw alone, too)
    w.check(got, start)
    want = r["dw"] + (start.double() if add else 0)
    logit = (D / 16 + 2) * 2 * U32 * r["S"]
    p_off = 2 * (logit + 16 * U32 * (1 + r["lse"].abs() + r["S"])) + 8 * U32 * (1 + r["lse"].abs())
    size = r["size"].T
    cost = (p_off * size + size * (2.0 ** -16 + (T / 16 + 64) * 2 * U32)) @ w.x.double().abs() + 2.0 ** -123 * w.x.double().abs().sum(0)
    assert ((got["dw"].double() - want).abs() <= cost + U16 * want.abs()).all()


def hot_rounding(w):
    """What rounding to bf16 takes from G at each row's target."""
    r = w.reference()
    hot = r["G"][torch.arange(w.T, device="cuda"), w.y.clamp(min=0)]
    return r, torch.where(w.y != -100, hot - hot.float().bfloat16().double(), 0.0)


@pytest.mark.parametrize("add,dx", [(False, True), (True, False)])
@pytest.mark.parametrize("T,V,D,chunk", [(257, 3000, 136, 0), (300, 4000, 136, 1024), (1500, 4000, 128, 0), (2100, 3000, 75, 0), (700, 300, 264, 0), (40000, 30000, 24, 0)])
def test_dw_gets_back_what_rounding_takes_from_g_at_the_target(T, V, D, chunk, add, dx):
    """As for dx, for rows of dw with one or two tokens: their remainders come back, sum over t of off_t x_t.  (Of more some or all are left;
    the last size has sums that leave the accumulators on the way.)"""
    w = World(T, V, D, bf16=True, bf16_dw=True, scale=0.7, vocab_chunk=chunk)
    if T > 10000:
        w.y[torch.rand(T, device="cuda") < 0.9] = -100
    start = (torch.randn(V, D, device="cuda") / (4 * T)).bfloat16() if add else None
    got = w.loss(accumulate=add, start=start, dx=dx)
    r, off = hot_rounding(w)
    many = torch.bincount(w.y.clamp(min=0)[w.y != -100], minlength=V) > 2
    lost = torch.zeros(V, D, device="cuda", dtype=torch.float64).index_add_(0, w.y.clamp(min=0), off[:, None] * w.x.double())
    lost[many] = 0
    want = r["dw"] + (start.double() if add else 0)
    share = float(((got["dw"].double() - want) * lost).sum() / lost.square().sum())
    assert abs(share) <= 0.25


def test_targets_of_many_rows():
    """More tokens of a target than are given back one by one, in whatever order their rows were met: the same bits each time, and within the bounds."""
    for targets in (1, 40, 150):
        w = World(900, 500, 72, bf16=True, bf16_dw=True)
        w.y = torch.where(w.y >= 0, w.y % targets, w.y)
        first = w.loss()
        w.check(first)
        for _ in range(5):
            again = w.loss()
            assert torch.equal(again["dw"], first["dw"]) and torch.equal(again["dx"], first["dx"])
        # the gradient apart
        w.op.forward(w.x, w.w, w.y)
        gw = torch.empty_like(first["dw"])
        w.op.backward(w.x, w.w, w.y, w.dlogp, None, None, gw)
        w.check(dict(first, dx=None, dw=gw))


def test_ignored_rows_are_in_no_target_s_list():
    """An ignored index inside the vocabulary, and targets outside it: nothing of such rows reaches dw but NaN from the latter."""
    w = World(300, 700, 72, bf16=True, bf16_dw=True, ignored=0.0, ignore_index=7)
    w.y[::3], w.y[1] = 7, 8
    got, r = w.loss(), head(w.x, w.w, w.y, 1.0, 7, w.dlogp)
    assert (got["dx"][::3] == 0).all()
    assert float((got["dw"].double() - r["dw"]).norm() / r["dw"].norm()) <= U16      # (each value is rounded by half a step at most, G's rest by less)
    w.y[4], w.y[5] = 700, -1
    got = w.loss()
    assert got["dw"].isnan().all() and got["dx"][4:6].isnan().all() and got["dx"][7:].isfinite().all()
