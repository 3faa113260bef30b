"""Outputs of the log probability entry points that meet another buffer of the call, and buffers off their elements, on the host:
each is refused before anything is enqueued."""
import pytest

INVALID = 1
ROWS, VOCAB, LD = 4, 100, 120


@pytest.fixture(scope="module")
def B():
    from paper_2505_05086_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def at(i):
    return (i + 1) << 40


def desc(B, dtype=0, top_k=0, ld=LD, ld_grad=LD):
    return B.LogprobDesc(dtype, top_k, ROWS, VOCAB, ld, ld_grad, -100, 1.0)


def overlaps(sizes, out, other):
    """Arguments in which output `out` and buffer `other` have a few bytes in common."""
    p = {n: at(i) for i, n in enumerate(sizes)}
    for shift in (0, sizes[other] - 8, 8 - sizes[out]):
        yield {**p, out: p[other] + shift}


STRIP = 4 * ((ROWS - 1) * LD + VOCAB)
F, I = 4 * ROWS, 8 * ROWS


@pytest.mark.parametrize("top_k", [0, 3])
def test_log_probabilities(B, top_k):
    L, d = B.lib(), desc(B, top_k=top_k)
    sizes = dict(logits=STRIP, targets=I, logp=F, entropy=F, lse=F)
    if top_k:
        sizes.update(top_logp=F * top_k, top_ids=I * top_k)
    outs = [n for n in sizes if n not in ("logits", "targets")]
    for out in outs:
        for other in sizes:
            if other == out:
                continue
            for p in overlaps(sizes, out, other):
                args = [p.get(n) for n in ("logits", "targets", "logp", "entropy", "lse", "top_logp", "top_ids")]
                assert L.asi_token_logprobs(d, *args, None) == INVALID, (out, other)


def test_gradient(B):
    L, d = B.lib(), desc(B)
    sizes = dict(targets=I, lse=F, entropy=F, dlogp=F, dentropy=F, dlogits=STRIP)
    for other in ("targets", "lse", "entropy", "dlogp", "dentropy"):
        for p in overlaps(sizes, "dlogits", other):
            assert L.asi_token_logprobs_grad(d, at(50), *p.values(), None) == INVALID, other
            p["logits"] = p["dlogits"]                               # over the logits row for row, and over the other too
            assert L.asi_token_logprobs_grad(d, p.pop("logits"), *p.values(), None) == INVALID, other


def test_loss(B):
    L, d = B.lib(), desc(B)
    sizes = dict(logits=STRIP, targets=I, dlogp=F, dentropy=F, logp=F, entropy=F, lse=F, dlogits=STRIP)
    for out in ("logp", "entropy", "lse", "dlogits"):
        for other in sizes:
            if other in (out, "logits") and out in (other, "dlogits"):
                continue
            for p in overlaps(sizes, out, other):
                assert L.asi_token_loss(d, *p.values(), None) == INVALID, (out, other)


def test_between_the_rows_and_not_quite(B):
    """A buffer that starts or ends in a row although the rest of it lies behind one."""
    L, x = B.lib(), at(50)
    for dtype, e in ((0, 4), (1, 2)):
        d, row, stride = desc(B, dtype, ld=130, ld_grad=130), VOCAB * e, 130 * e
        for shift in (row - 4, stride - F + 4, stride + row - 4, 3 * stride + row - 4, 4 - F):
            args = [x, at(1), at(2), at(3), x + shift // 4 * 4]
            assert L.asi_token_logprobs(d, *args, None, None, None) == INVALID, (dtype, shift)
            assert L.asi_token_loss(d, at(60), *[at(i) for i in range(1, 6)], x + shift // 4 * 4, x, None) == INVALID
            assert L.asi_token_logprobs_grad(d, at(60), at(1), x + shift // 4 * 4, at(3), at(4), at(5), x, None) == INVALID


def test_buffers_off_their_elements(B):
    """Values of 4 and 8 bytes that no kernel could read or write in one piece."""
    L, d, k = B.lib(), desc(B), desc(B, top_k=2)
    p = [at(i) for i in range(9)]
    for i, shift in ((1, 4), (2, 2), (3, 2), (4, 1), (5, 2), (6, 4)):              # targets, logp, entropy, lse, top_logp, top_ids
        q = [*p[:i], p[i] + shift, *p[i + 1:]]
        assert L.asi_token_logprobs(k, *q[:7], None) == INVALID, i
    for i, shift in ((1, 4), (2, 2), (3, 2), (4, 1), (5, 2)):                       # targets, lse, entropy, dlogp, dentropy
        q = [*p[:i], p[i] + shift, *p[i + 1:]]
        assert L.asi_token_logprobs_grad(d, *q[:7], None) == INVALID, i
    for i, shift in ((1, 4), (2, 2), (3, 2), (4, 1), (5, 2), (6, 3)):              # targets, dlogp, dentropy, logp, entropy, lse
        q = [*p[:i], p[i] + shift, *p[i + 1:]]
        assert L.asi_token_loss(d, *q[:8], None) == INVALID, i
    e = B.EmbeddingDesc(0, 1, 50, 16, 9, -1, 1.0)
    for shift in (1, 2, 4):
        assert L.asi_embedding_forward(e, at(0), at(1) + shift, at(2), None) == INVALID
        assert L.asi_embedding_wgrad(e, at(0) + shift, at(1), at(2), 0, at(3), L.asi_embedding_wgrad_ws_bytes(e), None) == INVALID
