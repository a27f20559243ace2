"""Sizes past 32 bits are refused in words before any call into the library, which would
take their low 32 bits (no GPU and no memory needed: tensors without storage)."""

import pytest

from test_lm_refusals import host  # noqa: F401 (a fixture)

torch = pytest.importorskip("torch")
FAR = (1 << 32) + 8


def far(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="meta")


def test_sizes_past_32_bits(host):  # noqa: F811
    losses, layers, made = host
    x, v = far(2, FAR), far(FAR)
    saved, one, t = far(2, 2), far(2), far(2, dtype=torch.int64)
    tall, targets = far(FAR, 2), far(FAR, dtype=torch.int64)
    calls = [lambda: layers.layer_norm(x), lambda: layers.layer_norm(x, v, v), lambda: layers.layer_norm(tall),
             lambda: layers.layer_norm_backward(x, x, v, saved), lambda: layers.layer_norm_backward(tall, tall, None, tall),
             lambda: layers.embedding(t, x), lambda: layers.embedding(t, tall), lambda: layers.embedding_backward(t, x, 4),
             lambda: layers.embedding_backward(t, far(2, 4), FAR), lambda: layers.embedding_backward(targets, tall, 4),
             lambda: losses.vocab_loss(x, x, t), lambda: losses.vocab_loss(tall, far(3, 2), targets),
             lambda: losses.vocab_loss(far(2, 2), tall, t), lambda: losses.vocab_logprobs(x, x, t), lambda: losses.vocab_logprobs(far(2, 2), tall, t),
             lambda: losses.vocab_logprobs_backward(x, x, t, saved, one), lambda: losses.vocab_workspace_bytes(x, x),
             lambda: losses.vocab_workspace_bytes(far(2, 2), tall), lambda: losses.token_logprobs(x, t),
             lambda: losses.workspace_bytes(x), lambda: layers.workspace_bytes(2, FAR), lambda: layers.workspace_bytes(FAR, 2),
             lambda: layers.workspace_bytes(2, 2, FAR), lambda: layers.workspace_bytes(1 << 66, 2)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="at most 2\\^31 - 1"):
            call()
            pytest.fail(f"call {i} went through")
    assert not made
    # the longest width that is taken, and one more
    assert layers.workspace_bytes(2, 1 << 24) > 0 and layers.workspace_bytes(2, (1 << 24) + 1) == 0
