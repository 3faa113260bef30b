"""Refusals of the token loss, embedding and AdamW entry points, on the host: no GPU is touched (a call that got as far as a
launch would report a CUDA error here)."""
import ctypes as C
import math

import pytest

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 4


@pytest.fixture(scope="module")
def B():
    from paper_2505_05086_b200 import build
    build.build()
    from paper_2505_05086_b200 import binding
    binding.lib()
    return binding


def at(i):
    return (i + 1) << 40


def logprob(B, **kw):
    d = dict(in_dtype=0, top_k=0, rows=4, vocab=100, ld=100, ld_grad=100, ignore_index=-100, scale=1.0)
    d.update(kw)
    return B.LogprobDesc(*[d[f] for f, _ in B.LogprobDesc._fields_])


@pytest.mark.parametrize("bad,code", [
    (dict(in_dtype=2), INVALID), (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(ld=99), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID),
    (dict(rows=(1 << 27) + 1), UNSUPPORTED), (dict(vocab=(1 << 30) + 1, ld=1 << 31), UNSUPPORTED), (dict(ld=1 << 62), INVALID),
])
def test_logprob_descriptors(B, bad, code):
    L, d = B.lib(), logprob(B, **bad)
    p = [at(i) for i in range(9)]
    assert L.asi_token_logprobs(d, *p[:5], None, None, None) == code
    assert L.asi_token_logprobs_grad(d, *p[:7], None) == code
    assert L.asi_token_loss(d, *p[:8], None) == code
    assert L.asi_token_logprobs(None, *p[:5], None, None, None) == INVALID


def test_logprob_pointers(B):
    L, d = B.lib(), logprob(B)
    p = [at(i) for i in range(9)]
    for hole in (0, 1, 2, 4):                                        # logits, targets, logp, lse
        q = list(p)
        q[hole] = None
        assert L.asi_token_logprobs(d, *q[:5], None, None, None) == INVALID
    assert L.asi_token_logprobs(d, p[0] + 2, *p[1:5], None, None, None) == INVALID     # off an element
    assert L.asi_token_logprobs(d, *p[:5], p[5], p[6], None) == INVALID                # outputs without top_k
    for k, code in ((-1, INVALID), (33, INVALID), (101, INVALID)):
        assert L.asi_token_logprobs(logprob(B, top_k=k, vocab=20 if k == 33 else 100), *p[:7], None) == code
    k = logprob(B, top_k=3)
    assert L.asi_token_logprobs(k, *p[:5], p[5], None, None) == INVALID
    assert L.asi_token_logprobs(k, *p[:5], None, p[6], None) == INVALID
    for hole in (0, 1, 2, 4, 6):
        q = list(p)
        q[hole] = None
        assert L.asi_token_logprobs_grad(d, *q[:7], None) == INVALID
    q = list(p)
    q[3] = None                                                      # entropy missing where dentropy is there
    assert L.asi_token_logprobs_grad(d, *q[:7], None) == INVALID
    for hole in (0, 1, 2, 4, 6, 7):
        q = list(p)
        q[hole] = None
        assert L.asi_token_loss(d, *q[:8], None) == INVALID


def test_gradients_over_the_logits(B):
    """dlogits may be the logits row for row, and nothing in between."""
    L, p = B.lib(), [at(i) for i in range(9)]

    def grad(d, dx):
        return L.asi_token_logprobs_grad(d, *p[:6], dx, None), L.asi_token_loss(d, *p[:7], dx, None)

    assert grad(logprob(B, ld_grad=99), p[8]) == (INVALID, INVALID)
    assert grad(logprob(B, ld_grad=104), p[0]) == (INVALID, INVALID)
    assert grad(logprob(B), p[0] + 4) == (INVALID, INVALID)
    assert grad(logprob(B), p[0] - 4) == (INVALID, INVALID)
    assert grad(logprob(B), p[0] + 4 * 399) == (INVALID, INVALID)
    assert grad(logprob(B), p[8] + 1) == (INVALID, INVALID)
    assert grad(logprob(B, ld=120), p[0] + 4 * 100) == (INVALID, INVALID)
    for shift in (99, 121, -99, 220 + 99, -220 - 99, 220):           # between its rows, and not quite
        assert grad(logprob(B, ld=220, ld_grad=220), p[0] + 4 * shift) == (INVALID, INVALID)


def test_empty_calls_do_nothing(B):
    L = B.lib()
    assert L.asi_token_logprobs(logprob(B, rows=0), *[None] * 8) == 0
    assert L.asi_token_logprobs_grad(logprob(B, rows=0), *[None] * 8) == 0
    assert L.asi_token_loss(logprob(B, rows=0), *[None] * 9) == 0
    assert L.asi_embedding_forward(embedding(B, tokens=0), *[None] * 4) == 0
    assert L.asi_adamw_step(adamw(B), None, 0, None) == 0
    assert L.asi_adamw_step(adamw(B), tensors(B, [dict(n=0)]), 1, None) == 0


def embedding(B, **kw):
    d = dict(table_dtype=0, in_dtype=1, vocab=50, dim=16, tokens=9, padding_idx=-1, scale=1.0)
    d.update(kw)
    return B.EmbeddingDesc(*[d[f] for f, _ in B.EmbeddingDesc._fields_])


@pytest.mark.parametrize("bad,code", [
    (dict(in_dtype=5), INVALID), (dict(vocab=0), INVALID), (dict(dim=0), INVALID), (dict(tokens=-1), INVALID),
    (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(padding_idx=50), INVALID), (dict(padding_idx=-2), INVALID),
    (dict(vocab=(1 << 30) + 1), UNSUPPORTED), (dict(dim=(1 << 22) + 1), UNSUPPORTED), (dict(tokens=(1 << 24) + 1), UNSUPPORTED),
])
def test_embedding_descriptors(B, bad, code):
    L, d = B.lib(), embedding(B, **bad)
    assert L.asi_embedding_forward(d, at(0), at(1), at(2), None) == code
    assert L.asi_embedding_wgrad(d, at(0), at(1), at(2), 0, at(3), 1 << 36, None) == code
    assert L.asi_embedding_wgrad_ws_bytes(d) == 0
    assert L.asi_embedding_forward(None, at(0), at(1), at(2), None) == INVALID
    assert L.asi_embedding_wgrad(None, at(0), at(1), at(2), 0, at(3), 1 << 36, None) == INVALID


def test_embedding_pointers_and_workspace(B):
    L, d = B.lib(), embedding(B)
    assert L.asi_embedding_forward(embedding(B, table_dtype=7), at(0), at(1), at(2), None) == INVALID
    for args in ((None, at(1), at(2)), (at(0), None, at(2)), (at(0), at(1), None), (at(0) + 2, at(1), at(2)), (at(0), at(1), at(2) + 1),
                 (at(0), at(1), at(0) + 64), (at(0), at(2) + 8, at(2))):
        assert L.asi_embedding_forward(d, *args, None) == INVALID
    need = L.asi_embedding_wgrad_ws_bytes(d)
    assert need >= 256 and need % 256 == 0
    for args in ((None, at(1), at(2)), (at(0), None, at(2)), (at(0), at(1), None), (at(0), at(1) + 1, at(2)), (at(0), at(1), at(2) + 2),
                 (at(0), at(2) + 256, at(2)), (at(2) + 64, at(1), at(2))):
        assert L.asi_embedding_wgrad(d, *args, 0, at(3), need, None) == INVALID
    assert L.asi_embedding_wgrad(d, at(0), at(1), at(2), 0, None, need, None) == INVALID
    assert L.asi_embedding_wgrad(d, at(0), at(1), at(2), 0, at(3), need - 1, None) == WORKSPACE
    assert L.asi_embedding_wgrad(d, at(0), at(1), at(2), 0, at(3) + 128, need, None) == WORKSPACE
    assert L.asi_embedding_wgrad(d, at(0), at(1), at(2), 0, at(2), need, None) == INVALID       # over dW
    assert L.asi_embedding_wgrad(d, at(0), at(3), at(2), 0, at(3), need, None) == INVALID       # over dOut


def test_a_workspace_serves_shorter_batches(B):
    L = B.lib()
    for dim in (1, 300):
        most = 0
        for T in list(range(0, 400)) + list(range(4000, 80000, 97)) + [4736, 4737, 9472, 9473, 37888, 37889]:
            need = L.asi_embedding_wgrad_ws_bytes(embedding(B, tokens=T, dim=dim, vocab=40000))
            bigger = L.asi_embedding_wgrad_ws_bytes(embedding(B, tokens=T + 1, dim=dim, vocab=40000))
            assert need <= bigger
            most = max(most, need)
        assert most <= L.asi_embedding_wgrad_ws_bytes(embedding(B, tokens=80000, dim=dim, vocab=40000))


def adamw(B, **kw):
    d = dict(weight_dtype=0, grad_dtype=1, state_bits=32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=1,
             lr_dev=None, step_dev=None, grad_scale=None)
    d.update(kw)
    return B.AdamwDesc(*[d[f] for f, _ in B.AdamwDesc._fields_])


def tensors(B, entries):
    arr = (B.AdamwTensor * len(entries))()
    for i, e in enumerate(entries):
        d = dict(weight=at(10 * i), grad=at(10 * i + 1), exp_avg=at(10 * i + 2), exp_avg_sq=at(10 * i + 3), exp_avg_scale=None,
                 exp_avg_sq_scale=None, copy=None, n=1000)
        d.update(e)
        for f, _ in B.AdamwTensor._fields_:
            setattr(arr[i], f, d[f])
    return arr


@pytest.mark.parametrize("bad", [
    dict(weight_dtype=2), dict(grad_dtype=-1), dict(state_bits=16), dict(lr=-1e-9), dict(lr=math.nan), dict(lr=math.inf),
    dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=9e-17), dict(eps=math.inf), dict(eps=1e300),
    dict(weight_decay=-1.0), dict(weight_decay=math.inf), dict(step=0), dict(lr_dev=at(99) + 2), dict(step_dev=at(99) + 4),
    dict(grad_scale=at(99) + 1), dict(lr=1e39), dict(weight_decay=1e39),
])
def test_adamw_descriptors(B, bad):
    assert B.lib().asi_adamw_step(adamw(B, **bad), tensors(B, [{}]), 1, None) == INVALID


def test_adamw_tensors(B):
    L = B.lib()

    def step(entries, n=None, **kw):
        return L.asi_adamw_step(adamw(B, **kw), tensors(B, entries), len(entries) if n is None else n, None)

    assert L.asi_adamw_step(None, tensors(B, [{}]), 1, None) == INVALID
    assert L.asi_adamw_step(adamw(B), None, 1, None) == INVALID
    assert step([{}], n=-1) == INVALID
    for hole in ("weight", "grad", "exp_avg", "exp_avg_sq"):
        assert step([{}, {hole: None}]) == INVALID
    assert step([dict(n=-1)]) == INVALID
    assert step([dict(weight=at(0) + 2)]) == INVALID
    assert step([dict(grad=at(1) + 1)]) == INVALID
    assert step([dict(copy=at(5) + 1)]) == INVALID
    assert step([{}], state_bits=8) == INVALID                                            # no scales
    assert step([dict(exp_avg_scale=at(5))], state_bits=8) == INVALID
    # written buffers that meet another buffer
    assert step([{}, dict(weight=at(0) + 3996)]) == INVALID
    assert step([{}, dict(weight=at(0))]) == INVALID
    assert step([dict(exp_avg_sq=at(2))]) == INVALID
    assert step([{}, dict(grad=at(0) + 100)]) == INVALID
    assert step([dict(copy=at(1))]) == INVALID
    assert step([dict(exp_avg_scale=at(2) + 999, exp_avg_sq_scale=at(6))], state_bits=8) == INVALID
    assert step([{}], grad_scale=at(0)) == INVALID
    assert step([{}], lr_dev=at(2) + 8) == INVALID
