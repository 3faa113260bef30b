"""Block ends (norm after a branch, gate, dropout, residual sum, next norm) and their gradients against the formulas in 64 bits."""
import itertools

import pytest
import torch

from tests.block_util import U16, U32, factors, norm

pytestmark = pytest.mark.gpu
DT = {True: torch.bfloat16, False: torch.float32}
EPS = 1e-5


class World:
    """Inputs of a block's end and what 64 bits make of them.  `gate`: rows that share a row of the gate, 0 for none."""

    def __init__(self, T, D, bf16=False, bf16_res=False, layer=False, after=True, gate=0, p=0.0, affine=True, h=True, shift=0, seed=0, rows=None):
        g = torch.Generator(device="cuda").manual_seed(1000 * T + D + seed)
        self.T, self.D, self.bf16, self.bf16_res, self.layer, self.after, self.gate_rows, self.p, self.shift = T, D, bf16, bf16_res, layer, after, gate, p, shift

        def normal(*s):
            return torch.randn(*s, generator=g, device="cuda")
        it, rt = DT[bf16], DT[bf16_res]
        self.y, self.h = self.buf(normal(T, D) + 0.3, it), self.buf(2 * normal(T, D), rt) if h else None
        self.dx, self.dh_out = self.buf(normal(T, D), it), self.buf(normal(T, D), rt)
        self.gate = self.buf(1 + 0.3 * normal(-(-T // gate), D), torch.float32) if gate else None
        vec = [self.buf(1 + 0.3 * normal(D), torch.float32) if affine else None, self.buf(0.3 * normal(D), torch.float32) if affine and layer else None,
               self.buf(1 + 0.3 * normal(D), torch.float32) if affine else None, self.buf(0.3 * normal(D), torch.float32) if affine and layer else None]
        self.aft, self.nxt = (tuple(vec[:2]) if after else (None, None)), tuple(vec[2:])
        from paper_2505_05086_b200.runner import ResidualNormRunner
        self.op = ResidualNormRunner(rows or T, D, bf16=bf16, bf16_residual=bf16_res, norm="layer" if layer else "rms", norm_after=after,
                                     rows_per_gate=gate, eps=EPS, res_scale=0.8, branch_scale=1.5, dropout=p, seed=99, stream_id=5)
        self.mask = factors(p, 99, 5, 3, T * D).view(T, D).cuda()

    def buf(self, x, dtype, fill=None):
        """A contiguous tensor, `shift` elements behind an aligned one."""
        flat = torch.zeros(x.numel() + self.shift, device="cuda", dtype=dtype)
        out = flat[self.shift:].view(x.shape)
        out.copy_(x)
        return out

    def forward(self, x=True):
        self.h_out, self.x = self.buf(torch.zeros(self.T, self.D), DT[self.bf16_res]), self.buf(torch.zeros(self.T, self.D), DT[self.bf16]) if x else None
        self.op.forward(self.y, self.h, self.h_out, self.x, gate=self.gate, after=self.aft, next=self.nxt, step=3)
        return self.h_out, self.x

    def reference(self):
        d = {k: v.double() if v is not None else None for k, v in dict(y=self.y, gate=self.gate, aw=self.aft[0], ab=self.aft[1], nw=self.nxt[0],
                                                                      nb=self.nxt[1]).items()}
        self.leaves = {k: v.requires_grad_(True) for k, v in d.items() if v is not None}
        z = norm(d["y"], self.layer, d["aw"], d["ab"], EPS) if self.after else d["y"]
        if self.gate is not None:
            z = z * d["gate"].repeat_interleave(self.gate_rows, 0)[:self.T]
        self.hl = (self.h.double() if self.h is not None else torch.zeros_like(z)).requires_grad_(True)
        h_out = 0.8 * self.hl + 1.5 * z * self.mask
        stored = self.h_out.double().requires_grad_(True)             # (the next norm reads what is stored)
        x = norm(stored, self.layer, d["nw"], d["nb"], EPS)
        return h_out, stored, x

    def grads(self, dx=True, dh_out=True, fill=None, accumulate=False):
        shapes = dict(dy=(self.y, DT[self.bf16]), dh=(self.y, DT[self.bf16_res]))
        out = {k: self.buf(torch.zeros(self.T, self.D), t) for k, (_, t) in shapes.items()}
        for k, v in (("gate", self.gate), ("aw", self.aft[0]), ("ab", self.aft[1]), ("nw", self.nxt[0] if dx else None), ("nb", self.nxt[1] if dx else None)):
            out["d" + k] = None if v is None else self.buf(torch.full(v.shape, 2.0 if accumulate else float("nan")), torch.float32)
        self.op.backward(self.y, self.h_out, self.dx if dx else None, self.dh_out if dh_out else None, out["dy"], out["dh"], gate=self.gate, after=self.aft,
                         next=self.nxt, dgate=out["dgate"], dafter=(out["daw"], out["dab"]), dnext=(out["dnw"], out["dnb"]), accumulate=accumulate, step=3)
        return out

    def reference_grads(self, dx=True, dh_out=True):
        h_out, stored, x = self.reference()
        up = self.dh_out.double() if dh_out else torch.zeros_like(h_out)
        out = {}
        if dx:
            names = [k for k in ("nw", "nb") if k in self.leaves]
            got = torch.autograd.grad((x * self.dx.double()).sum(), [stored] + [self.leaves[k] for k in names])
            up = up + got[0]
            out.update({"d" + k: v for k, v in zip(names, got[1:])})
        names = [k for k in ("y", "gate", "aw", "ab") if k in self.leaves]
        got = torch.autograd.grad((h_out * up).sum(), [self.hl] + [self.leaves[k] for k in names])
        out.update({"d" + k: v for k, v in zip(names, got[1:])}, dh=got[0])
        return out


def off(got, want, size=None):
    """Distance in norm, relative to that of the result, or of the terms that it is the difference of."""
    want = want.detach()
    return float((got.double() - want).norm() / (want if size is None else size).norm().clamp(min=1e-300))


def term_sizes(w):
    """dh and dy are differences d - n mean(d n) - mean d, times a deviation, of terms that may be much larger than they are (a norm over one
    value hardly depends on it: 1 - n^2 = eps / (y^2 + eps)).  Each term is rounded by itself, so an error goes by the terms' sizes."""
    def terms(d, x, wt):
        x = x.double()
        m = x.mean(1, keepdim=True) if w.layer else 0.0
        r = 1 / ((x - m).square().mean(1, keepdim=True) + EPS).sqrt()
        n, d = ((x - m) * r).abs(), d.abs() * (wt.double().abs() if wt is not None else 1)
        # (n itself is a difference of x and its mean)
        n = n + (m * r).abs() * 2.0 ** -6 if w.layer else n
        return r * (d + n * (d * n).mean(1, keepdim=True) + (d.mean(1, keepdim=True) if w.layer else 0))
    up = w.dh_out.double().abs() + terms(w.dx.double(), w.h_out, w.nxt[0])
    u = 1.5 * up * w.mask
    if w.gate is not None:
        u = u * w.gate.double().abs().repeat_interleave(w.gate_rows, 0)[:w.T]
    return dict(dh=0.8 * up, dy=terms(u, w.y, w.aft[0]) if w.after else u)


# fp32: about a dozen roundings a value, row sums whose error grows with the root of their length at most (8192 values: their partial sums
# of eight, of a warp and of the row are trees of 8 + 5 + 32 terms): 64 half steps.  Sums over T rows add T / 2 half steps at most where
# nothing cancels; random signs leave a norm sqrt(T) below the terms' sum, which the terms' own 64 half steps meet as well: 64 + sqrt(T).
def bound(bf16, T=0):
    return U16 if bf16 else (64 + T ** 0.5) * U32


SHAPES = [(1, 1), (2, 7), (3, 8), (5, 33), (9, 264), (40, 256), (300, 768), (77, 1000), (33, 2048), (10, 2056), (150, 3001), (12, 4096), (5, 5001), (4, 8192)]


@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("layer", [False, True])
def test_sizes(T, D, layer):
    if D == 1 and layer:
        pytest.skip("a layer norm over one value is its bias")
    for bf16, bf16_res in ((False, False), (True, False), (True, True)):
        w = World(T, D, bf16, bf16_res, layer, gate=max(1, T // 3), p=0.1)
        h_out, x = w.forward()
        want_h, _, want_x = w.reference()
        assert off(h_out, want_h) <= bound(bf16_res) and off(x, want_x) <= bound(bf16)
        got, want, size = w.grads(), w.reference_grads(), term_sizes(w)
        for k, v in want.items():
            if k in size:
                last = U16 * v if (bf16 if k == "dy" else bf16_res) else 0 * v
                assert float((got[k].double() - v).norm()) <= float(last.norm()) + 64 * U32 * float(size[k].norm()), (k, bf16, bf16_res)
            else:
                assert off(got[k], v) <= bound(False, T), (k, bf16, bf16_res)


@pytest.mark.parametrize("gate", [0, 1, 2, 5, 64, 1000])
@pytest.mark.parametrize("after,layer", [(True, False), (True, True), (False, True)])
@pytest.mark.parametrize("T,D", [(64, 264), (131, 40), (700, 96)])
def test_gates(gate, after, layer, T, D):
    """One row for a token, for a few, for more than there are; rows that workers share and rows of their own."""
    w = World(T, D, layer=layer, after=after, gate=gate, p=0.25)
    h_out, x = w.forward()
    want_h, _, want_x = w.reference()
    assert off(h_out, want_h) <= bound(False) and off(x, want_x) <= bound(False)
    got = w.grads()
    for k, v in w.reference_grads().items():
        assert off(got[k], v) <= bound(False, T), k
    added = w.grads(accumulate=True)
    for k, v in got.items():
        if k not in ("dy", "dh") and v is not None:
            assert torch.allclose(added[k], v + 2, rtol=4 * U32, atol=0), k


def test_parts_that_are_missing():
    for affine, h, dx, dh_out in itertools.product((True, False), repeat=4):
        if not dx and not dh_out:
            continue
        w = World(37, 96, layer=True, gate=9, affine=affine, h=h)
        h_out, x = w.forward()
        want_h, _, want_x = w.reference()
        assert off(h_out, want_h) <= bound(False) and off(x, want_x) <= bound(False)
        got = w.grads(dx, dh_out)
        for k, v in w.reference_grads(dx, dh_out).items():
            assert off(got[k], v) <= bound(False, 37), (k, affine, h, dx, dh_out)
    # no norm behind the sum: the same sum, and 0 for its statistics
    w = World(37, 96, gate=9)
    a = w.forward()[0]
    assert torch.equal(w.forward(x=False)[0], a) and (w.op.stats[:, 2:] == 0).all()


@pytest.mark.parametrize("shift", [1, 2, 4])
def test_buffers_off_16_bytes(shift):
    a, b = World(21, 264, True, False, True, gate=4, p=0.1), World(21, 264, True, False, True, gate=4, p=0.1, shift=shift)
    for u, v in zip(a.forward(), b.forward()):
        assert off(v, u.double()) <= U16
    want = a.reference_grads()
    got = b.grads()
    for k, v in want.items():
        assert off(got[k], v) <= bound(k == "dy", 21), k


def test_in_place():
    w = World(50, 264, gate=50, p=0.1)
    w.forward()
    want = w.grads()
    h = w.h.clone()
    w.op.forward(w.y, h, h, w.x, gate=w.gate, after=w.aft, next=w.nxt, step=3)
    assert torch.equal(h, w.h_out)
    dy, dh = w.dx.clone(), w.dh_out.clone()
    w.op.backward(w.y, w.h_out, dy, dh, dy, dh, gate=w.gate, after=w.aft, next=w.nxt, step=3)
    assert torch.equal(dy, want["dy"]) and torch.equal(dh, want["dh"])


def test_a_shorter_batch_leaves_the_rest():
    w = World(20, 264, gate=4, rows=50)
    w.op.stats.fill_(7)
    w.forward()
    assert (w.op.stats[20:] == 7).all() and not (w.op.stats[:20] == 7).any()
    got = w.grads()
    for k, v in w.reference_grads().items():
        assert off(got[k], v) <= bound(False, 20), k
    # nothing at all
    e = torch.empty(0, 264, device="cuda")
    w.op.forward(e, e, e, e, gate=torch.empty(0, 264, device="cuda"))
    d = torch.ones(264, device="cuda")
    w.op.backward(e, e, e, e, e, e, gate=torch.empty(0, 264, device="cuda"), dnext=(d, None))
    assert (d == 0).all()


def test_rows_without_spread_and_rows_of_nan():
    from paper_2505_05086_b200.runner import ResidualNormRunner
    for layer in (False, True):
        op = ResidualNormRunner(4, 96, norm="layer" if layer else "rms", norm_after=True, eps=EPS)
        y = torch.randn(4, 96, device="cuda")
        y[0], y[1] = 0.0, 3.0
        y[2, 5] = float("nan")
        h = torch.zeros(4, 96, device="cuda")
        h_out, x = torch.empty_like(h), torch.empty_like(h)
        op.forward(y, h, h_out, x)
        assert (h_out[0] == 0).all() and (x[0] == 0).all() and h_out[2].isnan().all() and x[2].isnan().all()
        if layer:
            assert (h_out[1] == 0).all() and abs(float(op.stats[1, 0]) - 3) <= 3 * 2.0 ** -20
        assert abs(float(op.stats[0, 1]) * EPS ** 0.5 - 1) <= 2.0 ** -20
        assert off(h_out[3:], norm(y[3:].double(), layer, None, None, EPS)) <= bound(False)
        dy, dh = torch.empty_like(h), torch.empty_like(h)
        op.backward(y, h_out, torch.ones_like(h), None, dy, dh)
        assert dy[[0, 1, 3]].isfinite().all() and dy[2].isnan().all()


def test_gradient_against_differences():
    """The whole function's slope along a random direction."""
    w = World(6, 40, layer=True, gate=2, p=0.2)
    w.forward()

    def value(t):
        s = {k: (v.double() + t * d if v is not None else None) for (k, v), d in zip(items, directions)}
        z = norm(s["y"], True, s["aw"], s["ab"], EPS) * s["gate"].repeat_interleave(2, 0)
        h = 0.8 * s["h"] + 1.5 * z * w.mask
        return (norm(h, True, s["nw"], s["nb"], EPS) * w.dx.double()).sum() + (h * w.dh_out.double()).sum()
    items = list(dict(y=w.y, h=w.h, gate=w.gate, aw=w.aft[0], ab=w.aft[1], nw=w.nxt[0], nb=w.nxt[1]).items())
    directions = [torch.randn_like(v, dtype=torch.float64) for _, v in items]
    slope = float(value(1e-5) - value(-1e-5)) / 2e-5
    got = w.grads()
    mine = sum(float((got["d" + k].double() * d).sum()) for (k, _), d in zip(items, directions))
    size = sum(float((got["d" + k].double() * d).abs().sum()) for (k, _), d in zip(items, directions))
    assert abs(mine - slope) <= (64 * U32 + 1e-8) * size              # (differences: 1e-10 of curvature, 1e-16 / 1e-5 of rounding)


def test_the_same_bits_again_on_another_stream_and_in_a_graph():
    w = World(500, 264, True, True, gate=30, p=0.1)
    w.forward()
    first = w.grads()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = w.grads()
    side.synchronize()
    step = torch.tensor([3], device="cuda")
    third = {k: None if v is None else torch.zeros_like(v) for k, v in first.items()}

    def go():
        w.op.forward(w.y, w.h, w.h_out, w.x, gate=w.gate, after=w.aft, next=w.nxt, step=step)
        w.op.backward(w.y, w.h_out, w.dx, w.dh_out, third["dy"], third["dh"], gate=w.gate, after=w.aft, next=w.nxt, dgate=third["dgate"],
                      dafter=(third["daw"], None), dnext=(third["dnw"], None), step=step)
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for v in third.values():
        if v is not None:
            v.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for k, v in first.items():
        if v is not None:
            assert torch.equal(second[k], v) and torch.equal(third[k], v), k
