"""What the runners of the token loss, embedding and AdamW hand to the library, on the CPU: its calls are replaced by a recorder,
streams and their events by stand-ins."""
import sys
import threading

import pytest
import torch


class Stream:
    """A stand-in for a stream: what it was made to wait for."""

    def __init__(self, handle):
        self.cuda_stream, self.device, self.waited = handle, torch.device("cpu"), []

    def wait_event(self, event):
        self.waited.append(event)

    def record_event(self):
        return f"event of {self.cuda_stream}"


class World:
    """The current stream, whether it is captured, and the calls that went out."""

    def __init__(self):
        self.home = self.now = Stream(0)
        self.captured = set()
        self.calls = []

    def __getitem__(self, name):
        return [args for n, args in self.calls if n == name]


class On:
    def __init__(self, world, stream):
        self.world, self.stream = world, stream

    def __enter__(self):
        self.before, self.world.now = self.world.now, self.stream or self.world.now

    def __exit__(self, *_):
        self.world.now = self.before


@pytest.fixture()
def world(monkeypatch):
    from paper_2505_05086_b200 import binding, build, runner
    build.build()
    w = World()
    monkeypatch.setattr(runner, "_cuda_device", lambda d: torch.device("cpu"))
    monkeypatch.setattr(runner, "_raw_stream", lambda index: w.now.cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    monkeypatch.setattr(torch.cuda, "device", lambda d: On(w, None))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: On(w, s))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: w.now)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: w.now.cuda_stream in w.captured)

    def recorder(name):
        return lambda *args: w.calls.append((name, args))

    for name in ("token_logprobs", "token_logprobs_grad", "token_loss", "embedding_forward", "embedding_wgrad", "adamw_step"):
        monkeypatch.setattr(binding, name, recorder(name))
    return w


class Buffer:
    """A stand-in for a buffer on the device: which streams the allocator was told of."""

    def __init__(self, like):
        self.like, self.told = like, []

    def record_stream(self, stream):
        self.told.append(stream.cuda_stream)

    def data_ptr(self):
        return self.like.data_ptr()

    def numel(self):
        return self.like.numel()


# ---- buffers and streams

def embedding(**kw):
    from paper_2505_05086_b200.runner import EmbeddingRunner
    return EmbeddingRunner(50, 8, 6, **kw)


def test_the_embedding_has_its_workspace_from_the_start(world):
    """Made within a call, it would come from the current stream's memory, or from that of a graph that is being captured."""
    from paper_2505_05086_b200 import binding
    r = embedding()
    assert r.ws is not None and r.ws.numel() == binding.embedding_wgrad_ws_bytes(binding.EmbeddingDesc(0, 0, 50, 8, 6, -1, 1.0)) > 0
    r.ws = ws = Buffer(r.ws)
    r.wgrad(torch.zeros(6, dtype=torch.int64), torch.zeros(6, 8), torch.zeros(50, 8), stream=Stream(7))
    assert r.ws is ws and world["embedding_wgrad"][0][5:7] == (ws.data_ptr(), ws.numel())


def test_another_stream_waits_for_the_buffers_and_the_allocator_learns_of_it(world):
    r = embedding()
    r.ws = Buffer(r.ws)
    ids, d, dw = torch.zeros(6, dtype=torch.int64), torch.zeros(6, 8), torch.zeros(50, 8)
    r.wgrad(ids, d, dw)
    assert r.ws.told == [] and world.home.waited == []               # the stream they were made on
    side = Stream(7)
    for _ in range(3):
        r.wgrad(ids, d, dw, stream=side)
    assert r.ws.told == [7] and side.waited == ["event of 0"]
    world.now = other = Stream(9)                                    # the current one, without an argument
    r.wgrad(ids, d, dw)
    assert r.ws.told == [7, 9] and other.waited == ["event of 0"]
    assert [c[-1] for c in world["embedding_wgrad"]] == [0, 7, 7, 7, 9]


def test_a_capture_does_not_wait_for_what_is_outside_it(world):
    r = embedding()
    r.ws = Buffer(r.ws)
    ids, d, dw = torch.zeros(6, dtype=torch.int64), torch.zeros(6, 8), torch.zeros(50, 8)
    side = Stream(7)
    world.captured.add(7)
    r.wgrad(ids, d, dw, stream=side)
    assert r.ws.told and not side.waited
    world.captured.clear()
    r.wgrad(ids, d, dw, stream=side)
    assert side.waited == ["event of 0"]


def test_results_and_states_are_lent_too(world):
    from paper_2505_05086_b200.runner import AdamWRunner, LogprobRunner
    r = LogprobRunner(4, 10, top_k=2)
    assert {id(x) for x in r._own()} == {id(x) for x in (r.logp, r.entropy, r.lse, r.top_logp, r.top_ids)}
    a = AdamWRunner([torch.zeros(300)], [torch.zeros(300)], bits8=True)
    assert {x.data_ptr() for x in a._own()} == {x[0].data_ptr() for x in (a.exp_avg, a.exp_avg_sq, a.exp_avg_scale, a.exp_avg_sq_scale)}
    given = [torch.zeros(300)]
    a = AdamWRunner([torch.zeros(300)], [torch.zeros(300)], exp_avg=given)
    assert [x.data_ptr() for x in a._own()] == [a.exp_avg_sq[0].data_ptr()]


# ---- threads

@pytest.fixture()
def impatient():
    before = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    yield
    sys.setswitchinterval(before)


def side_by_side(*jobs, times=10000):
    def repeat(job):
        for _ in range(times):
            job()
    threads = [threading.Thread(target=repeat, args=(job,)) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()


def test_threads_that_share_an_embedding_send_their_own_number_of_tokens(world, impatient, monkeypatch):
    from paper_2505_05086_b200 import binding
    from paper_2505_05086_b200.runner import EmbeddingRunner
    r = EmbeddingRunner(50, 8, 64)
    table, wrong = torch.zeros(50, 8), []
    batches = {n: (torch.zeros(n, dtype=torch.int64), torch.zeros(n, 8)) for n in (3, 64)}
    tokens = {ids.data_ptr(): n for n, (ids, _) in batches.items()}

    def call(desc, table, ids, out, stream):
        if desc.tokens != tokens[ids]:
            wrong.append(desc.tokens)

    monkeypatch.setattr(binding, "embedding_forward", call)
    side_by_side(*(lambda ids=ids, out=out: r.forward(table, ids, out) for ids, out in batches.values()))
    assert not wrong


def test_threads_that_share_a_token_loss_send_their_own_rows(world, impatient, monkeypatch):
    from paper_2505_05086_b200 import binding
    from paper_2505_05086_b200.runner import LogprobRunner
    r, wrong, rows = LogprobRunner(64, 10), [], {}

    def call(desc, logits, *_):
        if (desc.rows, desc.ld) != rows[logits]:
            wrong.append((desc.rows, desc.ld))

    monkeypatch.setattr(binding, "token_logprobs", call)
    jobs = []
    for n, ld in ((3, 10), (64, 17)):
        x, y = torch.zeros(n, ld)[:, :10], torch.zeros(n, dtype=torch.int64)
        rows[x.data_ptr()] = (n, ld)
        jobs.append(lambda x=x, y=y: r.forward(x, y))
    side_by_side(*jobs)
    assert not wrong


# ---- buffers that are exchanged

def token_loss_calls(r, world, n=3):
    x, y, w = torch.zeros(n, 10), torch.zeros(n, dtype=torch.int64), torch.ones(n)
    world.calls.clear()
    r.forward(x, y)
    r.loss(x, y, w, None, torch.zeros(n, 10))
    r.backward(x, y, w, w, torch.zeros(n, 10))
    f, l, b = (args for _, args in world.calls)
    return f[3:8], l[5:8], b[3:5]


@pytest.mark.parametrize("top_k", [0, 2])
def test_results_go_where_the_attributes_are(world, top_k):
    from paper_2505_05086_b200.runner import LogprobRunner
    r = LogprobRunner(4, 10, top_k=top_k)

    def check():
        tops = (r.top_logp.data_ptr(), r.top_ids.data_ptr()) if top_k else (0, 0)
        stats = (r.logp.data_ptr(), r.entropy.data_ptr(), r.lse.data_ptr())
        f, l, b = token_loss_calls(r, world)
        assert f == stats + tops and l == stats and b == (stats[2], stats[1])

    check()
    r.lse, r.entropy = torch.zeros(4), torch.zeros(7)                # another buffer, a longer one
    check()
    r.logp.data = torch.zeros(4)                                     # other memory beneath the same tensor
    check()
    if top_k:
        r.top_ids = torch.zeros(4, 2, dtype=torch.int64)
        r.top_logp.set_(torch.zeros(4, 2))
        check()


def test_results_that_could_not_be_written_are_refused(world):
    from paper_2505_05086_b200.runner import LogprobRunner
    r = LogprobRunner(4, 10, top_k=2)
    lse = r.lse
    for bad in (None, torch.zeros(4, dtype=torch.float64), torch.zeros(8)[::2], torch.zeros(4, 1), [0.0] * 4):
        with pytest.raises(ValueError):
            r.lse = bad
    with pytest.raises(ValueError):
        r.top_ids = torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        r.top_logp = torch.zeros(4, 3)
    assert r.lse is lse                                              # as it was
    with pytest.raises(ValueError):
        LogprobRunner(4, 10).top_ids = torch.zeros(4, 2, dtype=torch.int64)
    r.lse = torch.zeros(2)                                           # of a batch of two
    token_loss_calls(r, world, 2)
    with pytest.raises(ValueError):
        token_loss_calls(r, world, 3)
    r.lse = torch.zeros(4)
    r.lse.data = torch.zeros(4, dtype=torch.float64)
    with pytest.raises(ValueError):
        token_loss_calls(r, world, 3)
    r = LogprobRunner(4, 10)
    r.logp.untyped_storage().resize_(0)                              # no memory at all
    with pytest.raises(ValueError):
        token_loss_calls(r, world, 3)


def test_gradient_from_the_results_of_an_earlier_batch(world):
    from paper_2505_05086_b200.runner import LogprobRunner
    r = LogprobRunner(4, 10)
    x, y, w, out = torch.zeros(3, 10), torch.zeros(3, dtype=torch.int64), torch.ones(3), torch.zeros(3, 10)
    lse, h = torch.zeros(3), torch.zeros(3)
    r.backward(x, y, w, w, out, lse=lse, entropy=h)
    r.backward(x, y, w, None, out, lse=lse)
    assert [c[3:5] for c in world["token_logprobs_grad"]] == [(lse.data_ptr(), h.data_ptr()), (lse.data_ptr(), 0)]
    for kw in (dict(entropy=h), dict(lse=lse), dict(lse=lse[:2], entropy=h), dict(lse=lse.double(), entropy=h)):
        with pytest.raises(ValueError):
            r.backward(x, y, w, w, out, **kw)


def table_of(call):
    return [(e.weight, e.grad, e.exp_avg, e.exp_avg_sq, e.exp_avg_scale, e.exp_avg_sq_scale, e.copy, e.n) for e in call[1]]


def addresses(r):
    def at(x):
        return None if x is None else x.data_ptr()
    return [tuple(map(at, each)) + (each[0].numel(),) for each in zip(r.weights, r.grads, r.exp_avg, r.exp_avg_sq, r.exp_avg_scale,
                                                                      r.exp_avg_sq_scale, r.copies)]


@pytest.mark.parametrize("bits8", [False, True])
def test_steps_go_to_the_weights_and_gradients_where_they_lie(world, bits8):
    from paper_2505_05086_b200.runner import AdamWRunner
    ws, gs, cs = ([torch.zeros(300, dtype=t), torch.zeros(7, dtype=t)] for t in (torch.float32, torch.float32, torch.bfloat16))
    r = AdamWRunner(ws, gs, bits8=bits8, copies=cs)

    def check(step=r.step):
        step()
        assert table_of(world["adamw_step"][-1]) == addresses(r)

    check()
    ws[0].data = torch.ones(300)                                     # other memory beneath the same tensor
    check()
    gs[1].set_(torch.ones(7))
    check()
    cs[0].data = torch.ones(300, dtype=torch.bfloat16)
    check()
    r.exp_avg[1].data = torch.ones(7, dtype=r.exp_avg[1].dtype)      # a state: with rebind()
    r.rebind()
    check()


def test_memory_that_a_step_writes_stays_alive(world):
    """States that were exchanged without rebind(): the step goes to the old ones, which nobody else gets."""
    from paper_2505_05086_b200.runner import AdamWRunner
    w, g, m = torch.zeros(300), torch.zeros(300), torch.zeros(300)
    r = AdamWRunner([w], [g], exp_avg=[m])
    before = addresses(r)[0][2]
    m.data = torch.ones(300)
    r.step()
    assert table_of(world["adamw_step"][-1])[0][2] == before in {x.data_ptr() for x in r._kept}
    r.rebind()
    assert before not in {x.data_ptr() for x in r._kept}


def test_exchanges_that_could_not_be_stepped_are_refused(world):
    from paper_2505_05086_b200.runner import AdamWRunner
    ws, gs = [torch.zeros(300)], [torch.zeros(300)]
    r = AdamWRunner(ws, gs)
    for name in ("weights", "grads", "exp_avg", "exp_avg_sq"):       # silently without effect before
        with pytest.raises(AttributeError):
            setattr(r, name, [torch.zeros(300)])
        with pytest.raises(TypeError):
            getattr(r, name)[0] = torch.zeros(300)
    r.step()
    for bad in (torch.zeros(299), torch.zeros(300, dtype=torch.float64), torch.zeros(600)[::2]):
        gs[0].data = bad
        with pytest.raises(ValueError):
            r.step()
    gs[0].data = torch.zeros(300)
    r.step()
    ws[0].untyped_storage().resize_(0)                               # no memory at all
    with pytest.raises(ValueError):
        r.step()
    assert len(world["adamw_step"]) == 2


def test_weights_of_a_step_runner_lie_as_their_gradients(world):
    """A transposed weight has as many elements as dW, in another order."""
    from paper_2505_05086_b200.binding import Plan
    from paper_2505_05086_b200.runner import LayerRunner, StepRunner

    def layer(*a, **kw):
        r = LayerRunner.__new__(LayerRunner)
        r.plan = Plan(*a, **kw)
        r.dW = torch.zeros(r.plan.info.dw_elems)
        return r

    step = StepRunner.__new__(StepRunner)
    step.runners = [layer("linear", (4, 5, 12), (2, 2, 2), 10), layer("conv", (4, 6, 7, 8), (2, 2, 2, 2), 9, k=3, pad=1),
                    layer("conv", (4, 6, 7, 8), (2, 2, 2, 2), 6, k=3, groups=6), layer("conv", (4, 6, 7, 8), (2, 2, 2, 2), 9, k=1)]
    shapes = [(10, 12), (9, 6, 3, 3), (6, 1, 3, 3), (9, 6, 1, 1)]
    assert [tuple(r.dW_shape) for r in step.runners] == shapes
    good = [torch.zeros(s) for s in shapes]
    step.optimizer(good).step()
    step.optimizer([w.view(-1) for w in good]).step()
    step.optimizer([torch.zeros(2, 5, 12), torch.zeros(9, 54), torch.zeros(6, 9), torch.zeros(9, 6)]).step()
    for i, bad in ((0, (12, 10)), (0, (2, 60)), (1, (6, 9, 3, 3)), (1, (3, 3, 6, 9)), (3, (6, 9, 1, 1))):
        with pytest.raises(ValueError):
            step.optimizer([*good[:i], torch.zeros(bad), *good[i + 1:]])
    with pytest.raises(ValueError):
        step.optimizer(good[:3])


def test_steps_behind_one_that_the_device_counted(world):
    """Their number is on the device: going on from the last one given on the host would spoil the bias correction."""
    from paper_2505_05086_b200.runner import AdamWRunner
    r = AdamWRunner([torch.zeros(300)], [torch.zeros(300)])
    r.step(), r.step()
    r.step(step=torch.tensor([7]))
    with pytest.raises(ValueError):
        r.step()
    r.step(step=8)
    r.step()
    assert r.t == 9 and len(world["adamw_step"]) == 5


def test_scratch_of_a_cold_start_comes_from_the_stream_that_uses_it(world, monkeypatch):
    from types import SimpleNamespace
    from paper_2505_05086_b200.runner import LayerRunner
    seen, empty = [], torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: (seen.append(world.now.cuda_stream), empty(*a, **kw))[1])
    r = LayerRunner.__new__(LayerRunner)
    r.plan = SimpleNamespace(init_seeded_ws_bytes=lambda: 64, init_factors_seeded=lambda *a: seen.append(a[-1]))
    r.U, r.cur, r.core = [torch.zeros(4), torch.zeros(4)], 0, torch.zeros(4)
    r.init_factors_seeded(torch.zeros(4), 1, Stream(7))
    assert seen == [7, 7]
    r.ws_seed = None
    r.init_factors_seeded(torch.zeros(4), 1)
    assert seen == [7, 7, 0, 0]
