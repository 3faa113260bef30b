"""Output layer and loss without logits against the formulas in 64 bits."""
import pytest
import torch

from tests.block_util import U16, U32, head

pytestmark = pytest.mark.gpu
DT = {True: torch.bfloat16, False: torch.float32}


class World:
    def __init__(self, T, V, D, bf16=True, bf16_dw=True, scale=1.0, ent=False, seed=0, rows=None, ignored=0.15, **kw):
        from paper_2505_05086_b200.runner import HeadRunner
        g = torch.Generator(device="cuda").manual_seed(T + 1000 * V + D + seed)
        self.T, self.V, self.D, self.bf16, self.bf16_dw, self.scale = T, V, D, bf16, bf16_dw, scale
        self.x = torch.randn(T, D, generator=g, device="cuda").to(DT[bf16])
        self.w = (torch.randn(V, D, generator=g, device="cuda") * 2.5 / D ** 0.5).to(DT[bf16])
        self.y = torch.randint(0, V, (T,), generator=g, device="cuda")
        self.y[torch.rand(T, generator=g, device="cuda") < ignored] = -100
        self.dlogp = torch.randn(T, generator=g, device="cuda") / T
        self.dent = torch.randn(T, generator=g, device="cuda") / T if ent else None
        self.op = HeadRunner(rows or T, V, D, bf16=bf16, bf16_dw=bf16_dw, scale=scale, **kw)

    def loss(self, accumulate=False, dx=True, dw=True, start=None):
        gx = torch.full_like(self.x, float("nan")) if dx else None
        gw = (start.clone() if start is not None else torch.full((self.V, self.D), float("nan"), device="cuda", dtype=DT[self.bf16_dw])) if dw else None
        self.op.loss(self.x, self.w, self.y, self.dlogp, self.dent, gx, gw, accumulate=accumulate)
        return dict(logp=self.op.logp[:self.T].clone(), entropy=self.op.entropy[:self.T].clone(), lse=self.op.lse[:self.T].clone(), dx=gx, dw=gw)

    def reference(self):
        return head(self.x, self.w, self.y, self.scale, -100, self.dlogp, self.dent)

    def check(self, got, start=None):
        """Logits: products of 16 k add up at a time, and each of these sums is truncated (2^-23 of the row's |x| |w| sums at most): K / 16 of them, three
        terms (fp32) six times as many.  lse and logp then carry a dozen roundings of values of their size; entropy sums p |log p| on top.  G is off by its
        logit's error, relative, by roundings of its exponent (2^-24 of lse and of the logit each, twice) and by its own; its products are sums like the
        logits' of values no larger than sum |G| |w|, with G in bf16 (half a step of each) where the result is."""
        r = self.reference()
        steps = (self.D / 16 + 2) * (1 if self.bf16 else 6)
        logit = steps * 2 * U32 * r["S"]
        a = logit + 16 * U32 * (1 + r["lse"].abs() + r["S"])
        if not self.bf16:
            a = a + 8 * 2.0 ** -24 * r["S"]                           # (pairs of terms that are left out, 2^-24 each)
        assert ((got["lse"] - r["lse"]).abs() <= a).all()
        live = self.y != -100
        assert ((got["logp"] - r["logp"]).abs() <= 2 * a).all() and (got["logp"][~live] == 0).all()
        assert ((got["entropy"] - r["entropy"]).abs() <= 3 * a * (1 + r["entropy"])).all()
        p_off = (2 * a + 8 * U32 * (1 + r["lse"].abs()))[:, None]
        size = r["size"]
        for name, bf16, other, transposed in (("dx", self.bf16, self.w, False), ("dw", self.bf16_dw, self.x, True)):
            if got[name] is None:
                continue
            g = size.T if transposed else size
            q = (p_off * size).T if transposed else p_off * size
            k = (self.T if transposed else self.V) / 16 + 64
            cost = (q + g * (U16 if bf16 else k * (1 if self.bf16 and transposed else 6) * 2 * U32)) @ other.double().abs()
            want = r[name] + (start.double() if start is not None and name == "dw" else 0)
            # (a probability below fp32's smallest normal, 2^-126, is 0, and so are terms of G below it: four times that at most, of weights up to 2)
            cost = cost + 2.0 ** -123 * other.double().abs().sum(0)
            last = (U16 if bf16 else 2 * U32) * want.abs()
            if bf16:
                cost = cost + (g * k * 2 * U32) @ other.double().abs()
            assert ((got[name].double() - want).abs() <= cost + last).all(), name


SIZES = [(1, 1, 1), (1, 2, 8), (2, 255, 7), (3, 256, 64), (5, 257, 65), (127, 300, 72), (128, 1000, 128), (129, 515, 200), (257, 770, 33), (300, 4000, 136), (9, 20000, 264),
         (600, 513, 1100)]


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("bf16,bf16_dw", [(True, True), (True, False), (False, False)])
@pytest.mark.parametrize("ent", [False, True])
def test_sizes_and_types(T, V, D, bf16, bf16_dw, ent):
    w = World(T, V, D, bf16, bf16_dw, scale=0.7, ent=ent)
    got = w.loss()
    w.check(got)
    assert w.op.device_status() == 0
    again = w.loss()
    for k, v in got.items():
        assert torch.equal(v, again[k]), k


@pytest.mark.parametrize("bf16,bf16_dw", [(True, True), (True, False), (False, False)])
@pytest.mark.parametrize("T,V,D", [(130, 1100, 136), (700, 2001, 75), (40, 3000, 520)])
def test_pieces_of_the_vocabulary(T, V, D, bf16, bf16_dw):
    """Five pieces and more, added to a gradient that is there: what a call with kept logits gives, to rounding."""
    for chunk in (1, 512):
        w = World(T, V, D, bf16, bf16_dw, ent=True, vocab_chunk=chunk)
        start = torch.randn(V, D, device="cuda").mul_(1 / T).to(DT[bf16_dw])
        w.check(w.loss(accumulate=True, start=start), start)
        one = World(T, V, D, bf16, bf16_dw, ent=True)
        a, b = w.loss(), one.loss()
        for k in ("logp", "entropy", "lse"):
            assert torch.equal(a[k], b[k]), k
        assert torch.equal(a["dw"], b["dw"])                          # (each row of dw comes from one piece)


def test_forward_and_backward_one_after_the_other():
    for bf16, bf16_dw in ((True, True), (False, False)):
        w = World(200, 1500, 136, bf16, bf16_dw, scale=1.3, ent=True)
        want = w.loss()
        gx, gw = torch.empty_like(w.x), torch.empty_like(want["dw"])
        w.op.forward(w.x, w.w, w.y)
        for k in ("logp", "entropy", "lse"):
            assert torch.equal(getattr(w.op, k), want[k])
        w.op.backward(w.x, w.w, w.y, w.dlogp, w.dent, gx, gw)
        w.check(dict(want, dx=gx, dw=gw))
        lse, ent = w.op.lse.clone(), w.op.entropy.clone()
        w.op.lse.fill_(0), w.op.entropy.fill_(0)
        only_x, only_w = torch.empty_like(gx), torch.empty_like(gw)
        w.op.backward(w.x, w.w, w.y, w.dlogp, w.dent, only_x, None, lse=lse, entropy=ent)
        w.op.backward(w.x, w.w, w.y, w.dlogp, w.dent, None, only_w, lse=lse, entropy=ent)
        assert torch.equal(only_x, gx) and torch.equal(only_w, gw)


def test_a_workspace_without_room_for_kept_logits_gives_the_same_bits():
    from paper_2505_05086_b200 import binding
    for bf16, bf16_dw in ((True, True), (True, False), (False, False)):
        w = World(70, 900, 136, bf16, bf16_dw, ent=True)
        want = w.loss()
        d = binding.HeadDesc.from_buffer_copy(w.op.desc)
        d.vocab_chunk = 900
        small = binding.head_ws_bytes(d, True)
        assert small < w.op.ws.numel()
        w.op.ws = torch.empty(small, dtype=torch.uint8, device="cuda")
        got = w.loss()
        for k in ("logp", "entropy", "lse", "dw", "dx"):
            assert torch.equal(got[k], want[k]), k


def test_rows_of_every_kind():
    """Ignored targets, targets outside, hidden states of NaN and infinity."""
    w = World(40, 700, 72, ignored=0.0, bf16_dw=True)
    w.y[3], w.y[4], w.y[5] = -100, 700, -1
    w.x[7, 2], w.x[8, 3] = float("nan"), float("inf")
    got = w.loss()
    assert got["logp"][3] == 0 and (got["dx"][3] == 0).all() and got["lse"][3].isfinite()
    for t in (4, 5):
        assert got["logp"][t].isnan() and got["dx"][t].isnan().all() and got["lse"][t].isfinite()
    for t in (7, 8):
        assert got["logp"][t].isnan() and got["lse"][t].isnan() and got["entropy"][t].isnan() and got["dx"][t].isnan().all()
    assert got["dw"].isnan().all()                                    # every row has a share of such a row
    fine = [t for t in range(40) if t not in (3, 4, 5, 7, 8)]
    clean = World(40, 700, 72, ignored=0.0, bf16_dw=True)
    want = clean.loss()
    for k in ("logp", "lse", "entropy", "dx"):
        assert torch.equal(got[k][fine], want[k][fine]), k
    # nothing but ignored rows
    w = World(40, 700, 72, bf16_dw=False)
    w.y.fill_(-100)
    got = w.loss()
    assert (got["logp"] == 0).all() and (got["dx"] == 0).all() and (got["dw"] == 0).all()


def test_an_ignored_index_inside_the_vocabulary():
    w = World(60, 300, 64, bf16=False, bf16_dw=False, ignored=0.0, ignore_index=7)
    w.y[::3] = 7
    got = w.loss()
    r = head(w.x, w.w, w.y, 1.0, 7, w.dlogp)
    assert (got["logp"][::3] == 0).all() and (got["dx"][::3] == 0).all()
    assert float((got["dw"].double() - r["dw"]).norm() / r["dw"].norm()) <= 2.0 ** -16


def test_large_logits():
    """Sums of exponentials that would overflow without the maximum, and rows whose first tiles are far below it."""
    w = World(20, 3000, 64, bf16=False, bf16_dw=False, ignored=0.0)
    w.x.mul_(40)
    w.w[:2000].mul_(0.01)
    got = w.loss()
    assert all(got[k].isfinite().all() for k in got)
    w.check(got)


def test_shorter_batches_and_none():
    w = World(90, 600, 72, rows=300)
    for k in ("logp", "entropy", "lse"):
        getattr(w.op, k).fill_(5)
    w.check(w.loss())
    for k in ("logp", "entropy", "lse"):
        assert (getattr(w.op, k)[90:] == 5).all()
    e, dw = torch.empty(0, 72, device="cuda", dtype=torch.bfloat16), torch.ones(600, 72, device="cuda", dtype=torch.bfloat16)
    y, f = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    w.op.loss(e, w.w, y, f, None, e.clone(), dw, accumulate=True)
    assert (dw == 1).all()
    w.op.loss(e, w.w, y, f, None, e.clone(), dw)
    assert (dw == 0).all()
    # hidden states of several dimensions, targets alike
    w = World(24, 600, 72)
    want = w.loss()
    gx, gw = torch.empty(4, 6, 72, device="cuda", dtype=torch.bfloat16), torch.empty_like(want["dw"])
    w.op.loss(w.x.view(4, 6, 72), w.w, w.y.view(4, 6), w.dlogp, None, gx, gw)
    assert torch.equal(gx.view(24, 72), want["dx"]) and torch.equal(gw, want["dw"])


def test_gradient_against_differences():
    w = World(12, 90, 20, bf16=False, bf16_dw=False, ent=True, scale=0.9)
    got = w.loss()
    dx, dw = torch.randn_like(w.x), torch.randn_like(w.w)

    def value(t):
        r = head(w.x.double() + t * dx, w.w.double() + t * dw, w.y, 0.9, -100)
        live = w.y != -100
        return float((r["logp"] * w.dlogp)[live].sum() + (r["entropy"] * w.dent)[live].sum())
    slope = (value(1e-5) - value(-1e-5)) / 2e-5
    mine = float((got["dx"].double() * dx).sum() + (got["dw"].double() * dw).sum())
    size = float((got["dx"].double() * dx).abs().sum() + (got["dw"].double() * dw).abs().sum())
    assert abs(mine - slope) <= (256 * U32 + 1e-8) * size


def test_two_runners_at_once_and_graphs():
    a, b = World(260, 3000, 136, ent=True, seed=1), World(260, 3000, 136, ent=True, seed=2)
    want = a.loss(), b.loss()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        one = a.loss()
        with torch.cuda.stream(side):
            two = b.loss()
        torch.cuda.synchronize()
        for k in want[0]:
            assert torch.equal(one[k], want[0][k]) and torch.equal(two[k], want[1][k]), k
    gx, gw = torch.zeros_like(a.x), torch.zeros(3000, 136, device="cuda", dtype=torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.op.loss(a.x, a.w, a.y, a.dlogp, a.dent, gx, gw)
    for _ in range(2):
        gx.zero_(), gw.zero_(), a.op.logp.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gx, want[0]["dx"]) and torch.equal(gw, want[0]["dw"]) and torch.equal(a.op.logp, want[0]["logp"])


def test_waits_that_run_out_are_reported():
    """The test hook: barriers are armed and no copy is issued, so that waits expire (a millisecond); nothing faults, and the workspace serves again."""
    from paper_2505_05086_b200.binding import ASI_ERR_TIMEOUT, ASI_FLAG_TEST_EXPIRE_WAIT
    for bf16, bf16_dw in ((True, True), (True, False), (False, False)):
        w = World(300, 2000, 136, bf16, bf16_dw)
        want = w.loss()
        assert w.op.device_status() == 0
        w.op.desc.flags = ASI_FLAG_TEST_EXPIRE_WAIT
        w.loss()
        assert w.op.device_status() == ASI_ERR_TIMEOUT
        w.op.desc.flags = 0
        got = w.loss()
        assert w.op.device_status() == 0
        for k in want:
            assert torch.equal(got[k], want[k]), k


def test_an_ordinary_size_with_many_pieces():
    """More tiles than pairs of SMs, several pieces, both products in one launch."""
    w = World(2100, 24000, 328, ent=False, vocab_chunk=6000)
    got = w.loss()
    w.check(got)
    f = World(1000, 9000, 1032, bf16=False, bf16_dw=False, ent=True, vocab_chunk=4000)
    f.check(f.loss())


def test_many_rows_of_few_columns():
    """More rows than a grid's second dimension has places, their logits kept."""
    w = World(70000, 3, 8, bf16_dw=False)
    w.check(w.loss())
    w.op.forward(w.x, w.w, w.y)
    assert ((w.op.lse - head(w.x, w.w, w.y, 1.0, -100)["lse"]).abs() <= 2.0 ** -18).all()


@pytest.mark.parametrize("bf16,bf16_dw", [(True, True), (True, False), (False, False)])
def test_gradients_off_16_bytes(bf16, bf16_dw):
    for chunk in (0, 512):
        w = World(70, 1100, 72, bf16, bf16_dw, vocab_chunk=chunk)
        start = torch.randn(1100, 72, device="cuda").mul_(1 / 70).to(DT[bf16_dw])
        want = w.loss(accumulate=True, start=start)
        gx = torch.zeros(70 * 72 + 1, device="cuda", dtype=DT[bf16])
        gw = torch.zeros(1100 * 72 + 3, device="cuda", dtype=DT[bf16_dw])
        gw[3:].view(1100, 72).copy_(start)
        w.op.loss(w.x, w.w, w.y, w.dlogp, None, gx[1:].view(70, 72), gw[3:].view(1100, 72), accumulate=True)
        assert torch.equal(gx[1:].view(70, 72), want["dx"]) and torch.equal(gw[3:].view(1100, 72), want["dw"])
        assert gx[0] == 0 and (gw[:3] == 0).all()
