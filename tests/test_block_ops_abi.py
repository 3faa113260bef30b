"""Refusals of the dropout, block end and output layer entry points, on the host: no GPU is touched (a call that got as far as a launch
would report a CUDA error here)."""
import math

import pytest

INVALID, UNSUPPORTED, WORKSPACE, CUDA = 1, 2, 4, 5


@pytest.fixture(scope="module")
def B():
    from paper_2505_05086_b200 import binding, build
    build.build()
    binding.lib()
    return binding


@pytest.fixture()
def no_gpu():
    """For calls with addresses that are none, of which nothing is wrong but that: they go as far as a launch, which only a host without a GPU
    answers with an error."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("needs a host without a GPU")


def at(i):
    return (i + 1) << 40


# ---- dropout

def drop(B, **kw):
    d = dict(p=0.1, seed=1, stream_id=2, step=0, step_dev=None)
    d.update(kw)
    return B.Dropout(*[d[f] for f, _ in B.Dropout._fields_])


@pytest.mark.parametrize("bad", [dict(p=-1e-9), dict(p=1.0), dict(p=math.nan), dict(p=math.inf), dict(p=1 - 2.0 ** -18), dict(step=-1),
                                 dict(step_dev=at(9) + 4)])
def test_dropout_descriptors(B, bad):
    assert B.lib().asi_dropout(drop(B, **bad), 0, 100, at(0), None, at(1), None) == INVALID


def test_dropout_buffers(B):
    L, d = B.lib(), drop(B)
    assert L.asi_dropout(None, 0, 100, at(0), None, at(1), None) == INVALID
    assert L.asi_dropout(d, 2, 100, at(0), None, at(1), None) == INVALID
    assert L.asi_dropout(d, 0, -1, at(0), None, at(1), None) == INVALID
    assert L.asi_dropout(d, 0, (1 << 40) + 1, at(0), None, at(50), None) == UNSUPPORTED
    assert L.asi_dropout(d, 0, 0, None, None, None, None) == 0
    for x, r, o in ((None, None, at(1)), (at(0), None, None), (at(0) + 2, None, at(1)), (at(0), at(2) + 1, at(1)), (at(0), None, at(1) + 2),
                    (at(0), None, at(0) + 4), (at(0), None, at(0) - 396), (at(0), at(1) + 4, at(1)), (at(0), at(0) + 8, at(0)),
                    (at(0), at(0), at(0) + 4)):
        assert L.asi_dropout(d, 0, 100, x, r, o, None) == INVALID
    assert L.asi_dropout(drop(B, step_dev=at(1) + 8), 0, 100, at(0), None, at(1), None) == INVALID
    assert L.asi_dropout(drop(B, step_dev=at(0)), 0, 100, at(0), at(0), at(0), None) == INVALID


# ---- block ends

ROWS, DIM = 6, 40


def branch_desc(B, drop_=None, **kw):
    d = dict(in_dtype=1, res_dtype=0, norm=1, norm_after=1, rows=ROWS, dim=DIM, rows_per_gate=2, eps=1e-5, res_scale=1.0, branch_scale=1.0,
             drop=drop_ or drop(B))
    d.update(kw)
    return B.BranchDesc(*[d[f] for f, _ in B.BranchDesc._fields_])


def branch(B, **kw):
    b = B.Branch(*[at(i) for i in range(len(B.Branch._fields_))])
    for k, v in kw.items():
        setattr(b, k, v)
    return b


NEED = 1 << 30


def both(B, d, b):
    L = B.lib()
    return L.asi_branch_forward(d, b, None), L.asi_branch_backward(d, b, 0, at(60), NEED, None)


@pytest.mark.parametrize("bad,code", [
    (dict(in_dtype=2), INVALID), (dict(res_dtype=2), INVALID), (dict(in_dtype=0, res_dtype=1), INVALID), (dict(norm=2), INVALID),
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(rows_per_gate=-1), INVALID), (dict(eps=0.0), INVALID), (dict(eps=math.nan), INVALID),
    (dict(eps=math.inf), INVALID), (dict(res_scale=math.inf), INVALID), (dict(branch_scale=math.nan), INVALID),
    (dict(dim=8193), UNSUPPORTED), (dict(rows=(1 << 27) + 1), UNSUPPORTED),
])
def test_branch_descriptors(B, bad, code):
    d = branch_desc(B, **bad)
    assert both(B, d, branch(B)) == (code, code)
    assert B.lib().asi_branch_backward_ws_bytes(d) == 0
    assert both(B, branch_desc(B, drop(B, p=2.0)), branch(B)) == (INVALID, INVALID)
    assert both(B, None, branch(B)) == (INVALID, INVALID) and both(B, branch_desc(B), None) == (INVALID, INVALID)


def test_branch_buffers(B):
    L, d = B.lib(), branch_desc(B)
    for hole in ("y", "stats", "gate"):
        assert both(B, d, branch(B, **{hole: None})) == (INVALID, INVALID), hole
    assert L.asi_branch_forward(d, branch(B, h_out=None), None) == INVALID
    for holes in (("dy",), ("h_out",), ("dx", "dh_out"), ("dx",)):       # (without dx, sums of the next norm have nothing to come from)
        assert L.asi_branch_backward(d, branch(B, **dict.fromkeys(holes)), 0, at(60), NEED, None) == INVALID, holes
    assert both(B, branch_desc(B, norm_after=0), branch(B)) == (INVALID, INVALID)
    plain = dict(after_weight=None, after_bias=None, dafter_weight=None, dafter_bias=None)
    for name in ("dafter_weight", "dafter_bias"):
        assert L.asi_branch_backward(branch_desc(B, norm_after=0), branch(B, **{**plain, name: at(50)}), 0, at(60), NEED, None) == INVALID
    assert L.asi_branch_backward(branch_desc(B, rows_per_gate=0), branch(B), 0, at(60), NEED, None) == INVALID     # dgate without a gate
    for name, shift in (("y", 1), ("h", 2), ("gate", 2), ("after_weight", 1), ("next_bias", 2), ("h_out", 2), ("x", 1), ("stats", 2)):
        assert L.asi_branch_forward(d, branch(B, **{name: at(30) + shift}), None) == INVALID, name
    for name, shift in (("y", 1), ("h_out", 2), ("dx", 1), ("dh_out", 2), ("dy", 1), ("dh", 2), ("dgate", 2), ("dnext_bias", 1)):
        assert L.asi_branch_backward(d, branch(B, **{name: at(30) + shift}), 0, at(60), NEED, None) == INVALID, name


def test_root_mean_square_norms_have_no_biases(B):
    L, d = B.lib(), branch_desc(B, norm=0)
    none = dict(after_bias=None, next_bias=None, dafter_bias=None, dnext_bias=None)
    for name in ("after_bias", "next_bias"):
        assert both(B, d, branch(B, **{**none, name: at(50)})) == (INVALID, INVALID)
    for name in ("dafter_bias", "dnext_bias"):
        assert L.asi_branch_backward(d, branch(B, **{**none, name: at(50)}), 0, at(60), NEED, None) == INVALID


def sizes(forward):
    n, w = ROWS * DIM, 4 * DIM
    s = dict(y=2 * n, gate=3 * w, after_weight=w, after_bias=w, next_weight=w, stats=16 * ROWS)
    s.update(dict(h=4 * n, next_bias=w, h_out=4 * n, x=2 * n) if forward else
             dict(h_out=4 * n, dx=2 * n, dh_out=4 * n, dy=2 * n, dh=4 * n, dgate=3 * w, dafter_weight=w, dafter_bias=w, dnext_weight=w, dnext_bias=w))
    return s


@pytest.mark.parametrize("forward", [True, False])
def test_branch_outputs_that_meet_another_buffer(B, forward):
    L, d, s = B.lib(), branch_desc(B), sizes(forward)
    outs = ("h_out", "x", "stats") if forward else ("dy", "dh", "dgate", "dafter_weight", "dafter_bias", "dnext_weight", "dnext_bias")
    over = {("h_out", "h"), ("dy", "dx"), ("dh", "dh_out")}            # row for row they may
    for out in outs:
        for other in s:
            if other == out:
                continue
            where = {n: at(i) for i, n in enumerate(s)}
            for shift in (0, s[other] - 4, 4 - s[out]):
                if shift == 0 and (out, other) in over:
                    continue
                b = branch(B, **{**where, out: where[other] + shift})
                got = L.asi_branch_forward(d, b, None) if forward else L.asi_branch_backward(d, b, 0, at(60), NEED, None)
                assert got == INVALID, (out, other, shift)
    step = branch_desc(B, drop(B, step_dev=at(2)))
    b = branch(B, **{"x" if forward else "dy": at(2) - 8})
    assert (L.asi_branch_forward(step, b, None) if forward else L.asi_branch_backward(step, b, 0, at(60), NEED, None)) == INVALID


def test_branch_workspace(B):
    L, d = B.lib(), branch_desc(B)
    need = L.asi_branch_backward_ws_bytes(d)
    assert need > 0 and need % 256 == 0
    assert L.asi_branch_backward(d, branch(B), 0, None, need, None) == INVALID
    assert L.asi_branch_backward(d, branch(B), 0, at(60), need - 1, None) == WORKSPACE
    assert L.asi_branch_backward(d, branch(B), 0, at(60) + 128, need, None) == WORKSPACE
    assert L.asi_branch_backward(d, branch(B, dy=at(60)), 0, at(60), need, None) == INVALID
    for dim in (1, 300, 2048, 5000, 8192):
        most = 0
        for rows in list(range(0, 700)) + [1000, 4096, 5000, 100000]:
            n = L.asi_branch_backward_ws_bytes(branch_desc(B, rows=rows, dim=dim))
            assert n >= most
            most = n


def test_branch_empty_calls_do_nothing(B):
    L, d = B.lib(), branch_desc(B, rows=0)
    empty = B.Branch()
    assert L.asi_branch_forward(d, empty, None) == 0
    assert L.asi_branch_backward(d, empty, 0, None, 0, None) == 0
    assert L.asi_branch_backward(d, branch(B), 1, None, 0, None) == 0


# ---- output layer and loss

T, V, D = 5, 300, 24


def head_desc(B, **kw):
    d = dict(in_dtype=1, dw_dtype=0, rows=T, vocab=V, dim=D, vocab_chunk=0, ignore_index=-100, scale=1.0, flags=0)
    d.update(kw)
    return B.HeadDesc(*[d[f] for f, _ in B.HeadDesc._fields_])


ARGS = (("x", "w", "y", "logp", "entropy", "lse"), ("x", "w", "y", "lse", "entropy", "dlogp", "dent", "dx", "dw"),
        ("x", "w", "y", "dlogp", "dent", "logp", "entropy", "lse", "dx", "dw"))
FORWARD, GRAD, LOSS = range(3)


def call(B, k, d, p, ws=at(60), n=NEED):
    """The code of entry point k for buffers by name."""
    L = B.lib()
    args = [p.get(x) for x in ARGS[k]]
    if k == FORWARD:
        return L.asi_head_logprobs(d, *args, ws, n, None)
    return (L.asi_head_grad if k == GRAD else L.asi_head_loss)(d, *args, 0, ws, n, None)


def refused(B, d, p, code=INVALID, which=(FORWARD, GRAD, LOSS), **kw):
    """(No entry point is called that has nothing to refuse: it would go as far as a launch.)"""
    return all(call(B, k, d, p, **kw) == code for k in which)


NAMES = ("x", "w", "y", "dlogp", "dent", "logp", "entropy", "lse", "dx", "dw")


def buffers(**kw):
    return {**{n: at(i) for i, n in enumerate(NAMES)}, **kw}


@pytest.mark.parametrize("bad,code", [
    (dict(in_dtype=2), INVALID), (dict(dw_dtype=2), INVALID), (dict(in_dtype=0, dw_dtype=1), INVALID), (dict(rows=-1), INVALID),
    (dict(vocab=0), INVALID), (dict(dim=0), INVALID), (dict(vocab_chunk=-1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=math.nan), INVALID),
    (dict(scale=math.inf), INVALID), (dict(flags=1), INVALID), (dict(flags=6), INVALID), (dict(rows=(1 << 22) + 1), UNSUPPORTED),
    (dict(vocab=(1 << 24) + 1), UNSUPPORTED), (dict(dim=(1 << 16) + 1), UNSUPPORTED),
])
def test_head_descriptors(B, bad, code):
    d = head_desc(B, **bad)
    assert refused(B, d, buffers(), code)
    assert B.lib().asi_head_ws_bytes(d, 0) == B.lib().asi_head_ws_bytes(d, 1) == 0
    assert refused(B, None, buffers())


def test_head_buffers(B):
    d = head_desc(B)
    for hole in ("x", "w", "y"):
        assert refused(B, d, buffers(**{hole: None}))
    for hole, which in (("logp", (FORWARD, LOSS)), ("lse", (FORWARD, GRAD, LOSS)), ("dlogp", (GRAD, LOSS)), ("entropy", (GRAD, LOSS))):
        assert refused(B, d, buffers(**{hole: None}), which=which), hole      # (entropy missing where dentropy is there)
    assert refused(B, d, buffers(dx=None, dw=None), which=(GRAD, LOSS))
    for name, shift in (("x", 2), ("x", 8), ("w", 8), ("y", 4), ("logp", 2), ("lse", 1), ("entropy", 2), ("dlogp", 2), ("dent", 2), ("dx", 1), ("dw", 2)):
        which = [k for k in range(3) if name in ARGS[k]]                      # x and w on 16 bytes (dim 24)
        assert refused(B, d, buffers(**{name: at(30) + shift}), which=which), name
    assert refused(B, d, buffers(), ws=None)


def test_head_outputs_that_meet_another_buffer(B):
    d = head_desc(B)
    size = dict(x=2 * T * D, w=2 * V * D, y=8 * T, dlogp=4 * T, dent=4 * T, logp=4 * T, entropy=4 * T, lse=4 * T, dx=2 * T * D, dw=4 * V * D)
    writes = (("logp", "entropy", "lse"), ("dx", "dw"), ("logp", "entropy", "lse", "dx", "dw"))
    need = B.lib().asi_head_ws_bytes(d, 1)
    for k in range(3):
        for out in writes[k]:
            for other in ARGS[k]:
                for shift in (0, size[other] // 16 * 16 - 16, 16 - size[out] // 16 * 16):
                    p = buffers()
                    p[out] = p[other] + shift
                    if other != out and p[out] < p[other] + size[other] and p[other] < p[out] + size[out]:
                        assert refused(B, d, p, which=(k,)), (k, out, other, shift)
        for name in ARGS[k]:
            assert refused(B, d, buffers(**{name: at(60) + 256}), which=(k,), n=need), (k, name)


def test_head_workspace(B):
    L, d = B.lib(), head_desc(B, vocab_chunk=256)                       # (no logits are kept: all of it is needed)
    assert L.asi_head_ws_bytes(d, 0) < L.asi_head_ws_bytes(d, 1)
    for grad, which in ((0, (FORWARD,)), (1, (GRAD, LOSS))):
        need = L.asi_head_ws_bytes(d, grad)
        assert need % 256 == 0 and refused(B, d, buffers(), WORKSPACE, which, n=need - 1)
    assert refused(B, d, buffers(), WORKSPACE, ws=at(60) + 128)
    assert L.asi_head_ws_bytes(head_desc(B, vocab_chunk=256, vocab=100000, rows=4000), 1) < L.asi_head_ws_bytes(head_desc(B, vocab=100000, rows=4000), 1)


def test_room_for_kept_logits_is_not_insisted_on(B, no_gpu):
    L, kept = B.lib(), head_desc(B)
    assert L.asi_head_ws_bytes(kept, 1) > L.asi_head_ws_bytes(head_desc(B, vocab_chunk=V), 1)
    assert call(B, LOSS, kept, buffers(), n=L.asi_head_ws_bytes(head_desc(B, vocab_chunk=V), 1)) == CUDA


@pytest.mark.parametrize("kw", [dict(), dict(in_dtype=0), dict(dim=771), dict(vocab_chunk=1000), dict(in_dtype=1, dw_dtype=1)])
@pytest.mark.parametrize("vocab", [1, 5000, 130000])
def test_a_head_workspace_serves_fewer_rows(B, no_gpu, kw, vocab):
    """What fewer rows cannot do without fits (they may find room to keep their logits in as well, or not)."""
    L = B.lib()
    least = 0
    for rows in list(range(1, 300)) + [512, 1000, 1001, 4096, 4097, 8192, 20000]:
        d = head_desc(B, **{"vocab": vocab, "dim": 768, **kw, "rows": rows})
        n = L.asi_head_ws_bytes(d, 1)
        assert n >= least
        # found by bisection over the code that a call returns
        if rows in (1, 7, 256, 1000, 4097, 20000):
            lo, hi = 0, n
            p = dict(x=1 << 50, w=1 << 51, y=1 << 52, dlogp=1 << 53, logp=1 << 54, lse=1 << 55, dx=1 << 56, dw=1 << 57)
            while hi - lo > 256:
                mid = (lo + hi) // 512 * 256
                if call(B, LOSS, d, p, n=mid) == WORKSPACE:
                    lo = mid
                else:
                    hi = mid
            assert hi >= least
            least = hi


def test_head_without_rows(B):
    L, d = B.lib(), head_desc(B, rows=0)
    assert L.asi_head_logprobs(d, *[None] * 7, 0, None) == 0
    assert L.asi_head_grad(d, *[None] * 9, 0, None, 0, None) == 0
    assert L.asi_head_grad(d, *[None] * 8, at(0), 1, None, 0, None) == 0
    assert L.asi_head_loss(d, *[None] * 10, 0, None, 0, None) == 0
    assert L.asi_head_grad(d, *[None] * 8, at(0) + 2, 0, None, 0, None) == INVALID


def test_head_status(B):
    import ctypes as C
    assert B.lib().asi_head_status(None, None, C.byref(C.c_int32())) == INVALID
    assert B.lib().asi_head_status(at(0), None, None) == INVALID
