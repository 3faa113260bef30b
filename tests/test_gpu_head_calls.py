"""The output layer called in other ways: with and without room for logits that are kept, with no rows."""
import pytest
import torch

from tests.test_gpu_head import World

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,V,D,ent", [(70, 900, 1032, False), (70, 900, 1032, True), (300, 700, 136, False), (33, 1000, 2000, False)])
@pytest.mark.parametrize("bf16,bf16_dw", [(True, True), (True, False), (False, False)])
def test_kept_logits_and_logits_computed_again_give_the_same_bits(T, V, D, bf16, bf16_dw, ent):
    from paper_2505_05086_b200 import binding
    w = World(T, V, D, bf16, bf16_dw, ent=ent)
    want = w.loss()
    d = binding.HeadDesc.from_buffer_copy(w.op.desc)
    d.vocab_chunk = V
    small = binding.head_ws_bytes(d, True)
    assert small < w.op.ws.numel()
    w.op.ws = torch.empty(small, dtype=torch.uint8, device="cuda")
    got = w.loss()
    for k in want:
        if D <= 768 or not bf16_dw or k in ("logp", "entropy", "lse"):      # (G in bf16 goes by logits whose long sums are not segmented)
            assert torch.equal(got[k], want[k]), k
    w.check(got)


def none(w):
    """A call without rows."""
    e, y, f = torch.empty_like(w.x[:0]), w.y[:0], w.dlogp[:0]
    return dict(forward=lambda: w.op.forward(e, w.w, y),
                loss=lambda: w.op.loss(e, w.w, y, f, None, e.clone(), torch.zeros_like(w.w), accumulate=True),
                backward=lambda: w.op.backward(e, w.w, y, f, None, e.clone(), torch.zeros_like(w.w)))


@pytest.mark.parametrize("entry", ["forward", "loss", "backward"])
def test_the_status_of_a_call_without_rows(entry):
    """It is that call's own, behind one whose waits ran out (the test hook: no copies are issued, waits end after a millisecond) and as a runner's first."""
    from paper_2505_05086_b200.binding import ASI_ERR_TIMEOUT, ASI_FLAG_TEST_EXPIRE_WAIT
    w = World(40, 600, 72)
    w.op.desc.flags = ASI_FLAG_TEST_EXPIRE_WAIT
    w.loss()
    assert w.op.device_status() == ASI_ERR_TIMEOUT
    w.op.desc.flags = 0
    none(w)[entry]()
    assert w.op.device_status() == 0


def test_the_status_before_any_call():
    """Whatever was in the memory that the allocator hands out."""
    old = torch.full((32 << 20,), 0x5A, dtype=torch.uint8, device="cuda")
    del old
    assert World(40, 600, 72).op.device_status() == 0


def test_gradients_apart_captured_and_beside_another():
    """backward() in a graph whose inputs change between replays, rows with a large lse among them, while another runner's runs on its own stream."""
    a, b = World(300, 1500, 136, bf16=False, bf16_dw=False, ent=True, seed=1), World(300, 1500, 136, ent=True, seed=2)

    def grads(w):
        gx, gw = torch.empty_like(w.x), torch.empty(1500, 136, device="cuda", dtype=torch.bfloat16 if w.bf16_dw else torch.float32)
        w.op.backward(w.x, w.w, w.y, w.dlogp, w.dent, gx, gw)
        return gx, gw
    a.op.forward(a.x, a.w, a.y), b.op.forward(b.x, b.w, b.y)
    other = grads(b)
    gx, gw = torch.empty_like(a.x), torch.empty(1500, 136, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        a.op.forward(a.x, a.w, a.y)
        a.op.backward(a.x, a.w, a.y, a.dlogp, a.dent, gx, gw)
    side.wait_stream(torch.cuda.current_stream())
    for scale in (1.0, 60.0, 1.0):                                    # (at 60 |lse| is beyond 128 in most rows)
        a.x.mul_(scale)
        graph.replay()
        with torch.cuda.stream(side):
            beside = grads(b)
        torch.cuda.synchronize()
        assert (a.op.lse.abs().max() > 128) == (scale > 1)
        want = grads(a)
        assert torch.equal(gx, want[0]) and torch.equal(gw, want[1])
        assert torch.equal(beside[0], other[0]) and torch.equal(beside[1], other[1])
        a.check(dict(logp=a.op.logp, entropy=a.op.entropy, lse=a.op.lse, dx=gx, dw=gw))
        a.x.div_(scale)


@pytest.mark.parametrize("bf16,bf16_dw", [(True, True), (True, False), (False, False)])
def test_waits_of_a_gradient_apart_that_run_out_are_reported(bf16, bf16_dw):
    """The test hook again (barriers are armed and no copy is issued, waits end after a millisecond)."""
    from paper_2505_05086_b200.binding import ASI_ERR_TIMEOUT, ASI_FLAG_TEST_EXPIRE_WAIT
    w = World(300, 2000, 136, bf16, bf16_dw)
    w.op.forward(w.x, w.w, w.y)

    def grads():
        gx, gw = torch.empty_like(w.x), torch.empty(2000, 136, device="cuda", dtype=torch.bfloat16 if bf16_dw else torch.float32)
        w.op.backward(w.x, w.w, w.y, w.dlogp, None, gx, gw)
        return gx, gw
    want = grads()
    assert w.op.device_status() == 0
    w.op.desc.flags = ASI_FLAG_TEST_EXPIRE_WAIT
    grads()
    assert w.op.device_status() == ASI_ERR_TIMEOUT
    w.op.desc.flags = 0
    got = grads()
    assert w.op.device_status() == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
