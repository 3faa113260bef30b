"""What the runners of dropout, block ends and the output layer hand to the library, on the CPU: its calls are replaced by a recorder, streams
and their events by stand-ins."""
import pytest
import torch

from tests.test_step_runners import Buffer, Stream, world as plain_world  # noqa: F401


@pytest.fixture()
def world(plain_world, monkeypatch):  # noqa: F811
    from paper_2505_05086_b200 import binding

    def recorder(name):
        # (descriptors are read within the call)
        def read(a):
            return type(a).from_buffer_copy(a) if hasattr(a, "_fields_") else binding.Branch.from_buffer_copy(a) if isinstance(a, bytes) else a
        return lambda *args: plain_world.calls.append((name, tuple(map(read, args))))
    for name in ("dropout", "branch_forward", "branch_backward", "head_logprobs", "head_grad", "head_loss"):
        monkeypatch.setattr(binding, name, recorder(name))
    return plain_world


def test_dropout(world):
    from paper_2505_05086_b200.runner import DropoutRunner
    r = DropoutRunner(0.25, seed=(1 << 63) + 5, stream_id=7, bf16=True)
    x, out = torch.zeros(3, 8, dtype=torch.bfloat16), torch.zeros(3, 8, dtype=torch.bfloat16)
    r.forward(x, out, step=9)
    d, dtype, n, *at = world["dropout"][0]
    assert (d.p, d.seed, d.stream_id, d.step, d.step_dev) == (0.25, (1 << 63) + 5, 7, 9, None)
    assert (dtype, n) == (1, 24) and at == [x.data_ptr(), 0, out.data_ptr(), 0]
    step = torch.tensor([4])
    r.backward(x, out, step=step)
    assert world["dropout"][1][0].step_dev == step.data_ptr()
    r.forward(x, out, residual=out)                                   # (the step on the device is not kept)
    assert world["dropout"][2][0].step_dev is None and world["dropout"][2][4] == out.data_ptr()
    for a, b, kw in ((x.float(), out, {}), (x, out.float(), {}), (x, out[:2], {}), (x, torch.zeros(8, 3, dtype=torch.bfloat16).T, {}),
                     (x, out, dict(residual=x[:1])), (x, out, dict(step=torch.tensor([1.0]))), (x, out, dict(step=torch.tensor([1, 2])))):
        with pytest.raises((ValueError, RuntimeError)):
            r.forward(a, b, **kw)
    assert len(world["dropout"]) == 3


def branch_runner(**kw):
    from paper_2505_05086_b200.runner import ResidualNormRunner
    return ResidualNormRunner(10, 8, **{**dict(norm_after=True, rows_per_gate=4), **kw})


def test_block_ends(world):
    r = branch_runner()
    y, h, h_out, x, gate, w = torch.zeros(2, 3, 8), torch.zeros(2, 3, 8), torch.zeros(2, 3, 8), torch.zeros(2, 3, 8), torch.zeros(2, 8), torch.zeros(8)
    r.forward(y, h, h_out, x, gate=gate, after=(w, None), next=(w, None), step=3)
    d, b, _ = world["branch_forward"][0]
    assert (d.rows, d.dim, d.rows_per_gate, d.drop.step) == (6, 8, 4, 3)
    assert (b.y, b.h, b.h_out, b.x, b.gate, b.after_weight, b.after_bias, b.next_weight, b.stats) == (
        y.data_ptr(), h.data_ptr(), h_out.data_ptr(), x.data_ptr(), gate.data_ptr(), w.data_ptr(), None, w.data_ptr(), r.stats.data_ptr())
    dg = torch.zeros(2, 8)
    r.backward(y, h_out, x, None, y, h, gate=gate, dgate=dg, dnext=(w, None), accumulate=True)
    d, b, accumulate, ws, n, _ = world["branch_backward"][0]
    assert (b.dx, b.dh_out, b.dy, b.dh, b.dgate, b.dnext_weight, b.dafter_weight) == (
        x.data_ptr(), None, y.data_ptr(), h.data_ptr(), dg.data_ptr(), w.data_ptr(), None)
    assert accumulate and (ws, n) == (r.ws.data_ptr(), r.ws.numel())
    ok = dict(gate=gate)
    for bad in (lambda: r.forward(torch.zeros(11, 8), None, torch.zeros(11, 8), gate=torch.zeros(3, 8)),       # more rows than it was made for
                lambda: r.forward(torch.zeros(2, 3, 9), None, h_out, **ok), lambda: r.forward(y, h[:1], h_out, **ok),
                lambda: r.forward(y, h, h_out.bfloat16(), **ok), lambda: r.forward(y, h, h_out), lambda: r.forward(y, h, h_out, gate=gate[:1]),
                lambda: branch_runner(rows_per_gate=0).forward(y, h, h_out, gate=gate), lambda: r.forward(y, h, h_out, after=(w[:7], None), **ok),
                lambda: r.forward(y, h, h_out, next=(None, w.double()), **ok), lambda: r.backward(y, h_out, x, None, y[:1], **ok),
                lambda: r.backward(y, h_out, x, None, y, dgate=gate[:1], **ok), lambda: branch_runner(norm="batch")):
        with pytest.raises(ValueError):
            bad()
    r.stats = torch.zeros(5, 4)
    with pytest.raises(ValueError):
        r.forward(y, h, h_out, **ok)
    assert len(world["branch_forward"]) == len(world["branch_backward"]) == 1


def head_runner(**kw):
    from paper_2505_05086_b200.runner import HeadRunner
    return HeadRunner(6, 50, 8, **kw)


def test_output_layer(world):
    r = head_runner()
    x, w, y, f, dx, dw = torch.zeros(2, 2, 8), torch.zeros(50, 8), torch.zeros(2, 2, dtype=torch.int64), torch.zeros(4), torch.zeros(2, 2, 8), torch.zeros(50, 8)
    r.forward(x, w, y)
    assert world["head_logprobs"][0][0].rows == 4
    assert world["head_logprobs"][0][1:] == (x.data_ptr(), w.data_ptr(), y.data_ptr(), r.logp.data_ptr(), r.entropy.data_ptr(), r.lse.data_ptr(),
                                             r.ws.data_ptr(), r.ws.numel(), 0)
    r.loss(x, w, y, f.view(2, 2), None, dx, None, accumulate=True)
    assert world["head_loss"][0][1:] == (x.data_ptr(), w.data_ptr(), y.data_ptr(), f.data_ptr(), 0, r.logp.data_ptr(), r.entropy.data_ptr(),
                                         r.lse.data_ptr(), dx.data_ptr(), 0, True, r.ws.data_ptr(), r.ws.numel(), 0)
    lse = torch.zeros(4)
    r.backward(x, w, y, f, None, dx, dw, lse=lse)
    assert world["head_grad"][0][4:10] == (lse.data_ptr(), 0, f.data_ptr(), 0, dx.data_ptr(), dw.data_ptr())
    new = torch.zeros(6)
    r.lse = new
    r.backward(x, w, y, f, f, None, dw)
    assert world["head_grad"][1][4:8] == (new.data_ptr(), r.entropy.data_ptr(), f.data_ptr(), f.data_ptr())
    seven = torch.zeros(7, dtype=torch.int64)
    for bad in (lambda: r.forward(torch.zeros(7, 8), w, seven), lambda: r.forward(x[:1], w, y), lambda: r.forward(x, w[:49], y),
                lambda: r.forward(x, w, y.int()), lambda: r.forward(x.bfloat16(), w, y), lambda: r.loss(x, w, y, f[:3], None, dx, dw),
                lambda: r.loss(x, w, y, f, f.double(), dx, dw), lambda: r.loss(x, w, y, f, None, dx[:1], dw), lambda: r.loss(x, w, y, f, None, dx, dw.bfloat16()),
                lambda: r.backward(x, w, y, f, f, dx, dw, lse=lse), lambda: r.backward(x, w, y, f, None, dx, dw, entropy=lse),
                lambda: head_runner(grad=False).loss(x, w, y, f, None, dx, dw), lambda: setattr(r, "logp", torch.zeros(3, 2))):
        with pytest.raises(ValueError):
            bad()
    r.logp = torch.zeros(3)
    with pytest.raises(ValueError):
        r.forward(x, w, y)
    assert [len(world[n]) for n in ("head_logprobs", "head_loss", "head_grad")] == [1, 1, 2]


def test_another_stream_waits_for_their_buffers(world):
    r = head_runner()
    ws = r.ws = Buffer(r.ws)
    x, w, y = torch.zeros(4, 8), torch.zeros(50, 8), torch.zeros(4, dtype=torch.int64)
    r._buffers = ()                                                   # (plain tensors of the CPU know no streams)
    side = Stream(7)
    r._streams.discard(7)
    for _ in range(2):
        r._call(side, lambda *a: None)
    assert ws.told == [7] and side.waited == ["event of 0"]
    b = branch_runner()
    b.ws, b._stats = Buffer(b.ws), Buffer(b.stats)
    other = Stream(9)
    b._call(other, lambda *a: None)
    assert b.ws.told == b._stats.told == [9] and other.waited == ["event of 0"]
