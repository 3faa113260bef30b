"""The output layer called in other ways: with and without room for logits that are kept."""
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
