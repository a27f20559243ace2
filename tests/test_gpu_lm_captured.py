"""Differentiable forms of the language-model operators captured for their values alone, while
results of the same weights are alive."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["no_grad", "inference_mode"])
def test_values_alone(mode):
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1511_05946_amd import layers, losses
    N, V, T = 48, 200, 70
    W, g, b = (x.requires_grad_(True) for x in (torch.randn(V, N, device="cuda"), torch.ones(N, device="cuda"), torch.zeros(N, device="cuda")))
    tokens, targets = torch.randint(0, V, (T,), device="cuda"), torch.randint(0, V, (T,), device="cuda")

    def run(tokens=tokens, targets=targets):
        h = layers.layer_norm_autograd(layers.embedding_autograd(tokens, W), g, b)
        return (*losses.vocab_loss_autograd(h, W, targets), losses.vocab_logprobs_autograd(h, W, targets))

    alive = run(tokens.clone(), targets.clone())   # with gradients, on the default stream: a training step under way
    graph = torch.cuda.CUDAGraph()
    with getattr(torch, mode)(), torch.cuda.graph(graph):
        got = run()
    assert not any(x.requires_grad for x in got)
    for k in range(4):
        if k == 2:
            tokens.copy_(tokens.flip(0))
            targets.copy_(targets.roll(3))
        graph.replay()
        with torch.no_grad():
            want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), k
        junk = torch.randn(1 << 20, device="cuda").sum().item()
        assert junk == junk
    # the step goes on: its backward pass, and captured with gradients the calls are refused as before
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tokens + 1
        with pytest.raises(RuntimeError, match="embedding_autograd"):
            layers.embedding_autograd(tokens, W)
    alive[0].backward()
    assert W.grad is not None and torch.isfinite(W.grad).all()
