"""Outputs of the language-model operators in memory that their call reads are refused on the
GPU as well, where the arguments go straight to the library, and nothing is written."""

import pytest

pytestmark = pytest.mark.gpu


def test_shared_memory_is_refused():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1511_05946_amd import layers, losses
    R, N, V = 100, 12, 40
    h, w, u = torch.randn(R, N, device="cuda"), torch.randn(V, N, device="cuda"), torch.ones(N, device="cuda")
    room = torch.zeros(8192, device="cuda")
    t = torch.zeros(R, dtype=torch.int64, device="cuda")
    targets = room[:2 * R].view(torch.int64)
    rows, tall, pairs, vector = room[:R * N].view(R, N), room[:V * N].view(V, N), room[:2 * R].view(R, 2), room[:R]
    saved = layers.layer_norm(h, u, save=True).saved
    s = losses.vocab_logprobs(h, w, t, save=True).saved
    before = room.clone()
    for i, call in enumerate((
            lambda: layers.embedding(targets, w, out=rows), lambda: layers.embedding_backward(targets, h, V, grad_weight=tall),
            lambda: layers.layer_norm_backward(h, h, u, pairs, out=rows), lambda: layers.layer_norm_backward(h, h, u, pairs, grads=(room[:N], None)),
            lambda: losses.vocab_loss(h, w, targets, out=rows), lambda: losses.vocab_loss(h, w, t, weights=vector, grad_weight=tall),
            lambda: losses.vocab_logprobs_backward(h, w, t, pairs, vector, out=rows),
            lambda: losses.vocab_logprobs_backward(h, w, t, s, vector, grad_weight=tall),
            lambda: losses.vocab_logprobs_backward(h, w, t, s, h[:, 0].contiguous(), scale=room[:1], grad_weight=tall))):
        with pytest.raises(ValueError, match="overlaps"):
            call()
            pytest.fail(f"call {i} went through")
    # the workspace, too
    big = torch.zeros(losses.vocab_workspace_bytes(h, w) + layers.workspace_bytes(R, N, V), dtype=torch.uint8, device="cuda")
    inside = big[:4 * R * N].view(torch.float32).view(R, N)
    for call in (lambda: losses.vocab_loss(h, w, t, out=inside, workspace=big), lambda: losses.vocab_logprobs(inside, w, t, workspace=big),
                 lambda: layers.layer_norm_backward(h, h, u, saved, out=inside, workspace=big),
                 lambda: layers.embedding_backward(t, inside, V, workspace=big)):
        with pytest.raises(Exception, match="invalid argument"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(room, before) and (big == 0).all()
    # beside one another in one memory: as anywhere else
    both = torch.zeros(2, R, N, device="cuda")
    both[0] = h
    r = losses.vocab_loss(both[0], w, t, out=both[1])
    assert torch.equal(both[0], h) and torch.equal(r.grad_hidden, losses.vocab_loss(h, w, t).grad_hidden)
    g = h.clone()
    want = layers.layer_norm_backward(h, h, u, saved)
    got = layers.layer_norm_backward(h, g, u, saved, out=g)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
