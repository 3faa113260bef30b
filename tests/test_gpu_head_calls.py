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
