"""Weights of the output layer's gradient that are not contiguous, on the CPU: where their copy is made, and until when it lives."""
import weakref

import pytest
import torch

from tests.test_block_runners import head_runner, world  # noqa: F401
from tests.test_step_runners import Stream, world as plain_world  # noqa: F401


class Weights(torch.Tensor):
    """Notes the stream that was current when a copy of it was made, and the copy."""
    copies, now = [], None

    @classmethod
    def __torch_function__(cls, function, types, args=(), kwargs=None):
        with torch._C.DisableTorchFunctionSubclass():
            out = function(*args, **(kwargs or {}))
        if isinstance(out, torch.Tensor) and out.data_ptr() != args[0].data_ptr():
            cls.copies.append((cls.now(), out.data_ptr(), weakref.ref(out)))
        return out


@pytest.mark.parametrize("entry", ["loss", "backward"])
def test_copies_are_made_on_the_call_s_stream_and_live_until_it_is_queued(world, monkeypatch, entry):  # noqa: F811
    """A copy that the current stream makes is not there yet when another one reads it, and memory that is given back before the launch may be another's."""
    from paper_2505_05086_b200 import binding
    monkeypatch.setattr(Weights, "copies", [])
    monkeypatch.setattr(Weights, "now", lambda: world.now.cuda_stream)
    r = head_runner()
    r._streams.add(7)
    x, w, y, dx = torch.zeros(2, 2, 8), torch.zeros(50, 8), torch.zeros(2, 2, dtype=torch.int64), torch.zeros(2, 2, 8)
    logp, ent = torch.arange(4.0).view(2, 2).T.as_subclass(Weights), torch.ones(1).expand(2, 2).as_subclass(Weights)
    seen = []

    def call(*args):
        alive = {at: ref() for _, at, ref in Weights.copies}
        seen.append([alive[at].flatten().tolist() for at in args if isinstance(at, int) and alive.get(at) is not None])
    monkeypatch.setattr(binding, "head_loss", call)
    monkeypatch.setattr(binding, "head_grad", call)
    getattr(r, entry)(x, w, y, logp, ent, dx, None, stream=Stream(7))
    assert [s for s, _, _ in Weights.copies] == [7, 7]
    assert seen == [[[0.0, 2.0, 1.0, 3.0], [1.0] * 4]]
    # on the current stream, and contiguous weights, which are not copied
    getattr(r, entry)(x, w, y, logp, None, dx, None)
    getattr(r, entry)(x, w, y, torch.ones(2, 2).as_subclass(Weights), None, dx, None, stream=Stream(7))
    assert [s for s, _, _ in Weights.copies] == [7, 7, 0]
